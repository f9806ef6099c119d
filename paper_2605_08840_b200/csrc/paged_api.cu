// C ABI of the paged cache: argument checks and kernel sequencing.
#include <cmath>

#include "paged.cuh"
#include "restkv_handle.cuh"

namespace restkv {

static restkv_status make_cache(const restkv_paged* s, PagedCache* out) {
  if (!s) return RESTKV_ERR_INVALID_ARG;
  if (s->batch < 1 || s->n_q_heads < 1 || s->n_kv_heads < 1 || s->head_dim < 1) return RESTKV_ERR_INVALID_ARG;
  if (s->n_q_heads % s->n_kv_heads != 0) return RESTKV_ERR_INVALID_ARG;
  if (s->dtype != RESTKV_BF16 && s->dtype != RESTKV_F32) return RESTKV_ERR_INVALID_ARG;
  if (s->page_rows < kBlockRows || s->page_rows % kBlockRows != 0 || s->n_pages < 1 || s->table_width < 1) return RESTKV_ERR_INVALID_ARG;
  if (s->lengths_per_head != 0 && s->lengths_per_head != 1) return RESTKV_ERR_INVALID_ARG;
  if (!(s->softcap >= 0.f) || !std::isfinite(s->softcap)) return RESTKV_ERR_INVALID_ARG;
  PagedCache c{};
  c.batch = s->batch; c.Hq = s->n_q_heads; c.Hkv = s->n_kv_heads; c.G = c.Hq / c.Hkv; c.d = s->head_dim;
  c.scale = s->softmax_scale != 0.f ? s->softmax_scale : 1.0f / sqrtf((float)c.d);
  if (!(c.scale > 0.f) || !std::isfinite(c.scale)) return RESTKV_ERR_INVALID_ARG;
  if (c.d % 32 != 0 || c.d > 256) return RESTKV_ERR_UNSUPPORTED;
  c.softcap = fminf(s->softcap, 0x1p100f);   // so that logits over it keep all their bits in fp32; they would have to pass 2^88 to notice
  c.format = s->page_format;
  switch (s->page_format) {
    case RESTKV_PAGES_BF16:
    case RESTKV_PAGES_F32:
      if ((s->page_format == RESTKV_PAGES_F32) != (s->dtype == RESTKV_F32)) return RESTKV_ERR_UNSUPPORTED;
      c.row_bytes = c.d * (s->page_format == RESTKV_PAGES_F32 ? 4 : 2);
      c.block_bytes = kBlockRows * c.row_bytes;
      break;
    case RESTKV_PAGES_INT4:
      if ((s->group != 32 && s->group != 64 && s->group != 128) || c.d % s->group != 0) return RESTKV_ERR_INVALID_ARG;
      c.group = s->group;
      c.row_bytes = c.d / 2;
      c.block_bytes = kBlockRows * c.row_bytes + 64 * (c.d / c.group);
      break;
    default:
      return RESTKV_ERR_INVALID_ARG;
  }
  c.page_rows = s->page_rows; c.n_pages = s->n_pages; c.table_width = s->table_width; c.per_head = s->lengths_per_head;
  c.head_bytes = (long long)(c.page_rows / kBlockRows) * c.block_bytes;
  // rows, of a sequence and (16 at a time) of the pool, are counted in 32 bits; heads of a batch are a grid's second dimension
  if (c.capacity() > 0x7FFFFFFFll - kBlockRows) return RESTKV_ERR_UNSUPPORTED;
  if ((long long)c.n_pages * c.Hkv * c.page_rows > 0x7FFFFFFFll) return RESTKV_ERR_UNSUPPORTED;
  if ((long long)c.batch * c.Hkv > 65535) return RESTKV_ERR_UNSUPPORTED;
  *out = c;
  return RESTKV_OK;
}

static restkv_status check_tokens(const PagedCache& c, int n_tokens) {
  if (n_tokens < 1) return RESTKV_ERR_INVALID_ARG;
  // the tokens of a batch, and the query rows of a KV head rounded up to a tile of 256, are counted in 32 bits
  if ((long long)c.batch * n_tokens > 0x7FFFFFFFll || (long long)c.G * n_tokens > 0x7FFFFFFFll - 256) return RESTKV_ERR_UNSUPPORTED;
  return RESTKV_OK;
}

// The kernels that a call runs on: the tensor pipe for bf16 with the head_dims it has (kernel path 1 keeps off it), else fp32.
static bool on_tensor_pipe(const PagedCache& c, bool f32) { return !f32 && paged_mma_supported(c); }

static bool in_chunks(const PagedCache& c, bool f32) { return !f32 && paged_chunk_supported(c); }

// The most that any kernel that the shape can run on needs.  It never falls as n_tokens grows (each part rises with them and, once there,
// stays), so that a workspace for the most tokens serves calls of fewer.
static size_t attend_bytes(const PagedCache& c, bool f32, int sm_count) {
  size_t most = paged_simt_bytes(c, sm_count);   // what every call can run on
  if (!f32 && paged_mma_shape(c) && paged_mma_bytes(c, sm_count) > most) most = paged_mma_bytes(c, sm_count);
  if (!f32 && paged_chunk_shape(c) && paged_chunk_bytes(c, sm_count) > most) most = paged_chunk_bytes(c, sm_count);
  return align256(most);
}

static restkv_status make_rows(const restkv_rows* s, int heads, int n, int d, RowsView* out) {
  if (!s || !s->data || !aligned16(s->data)) return RESTKV_ERR_INVALID_ARG;
  *out = RowsView{s->data, s->stride_b, s->stride_h, s->stride_n};
  if (s->stride_b == 0 && s->stride_h == 0 && s->stride_n == 0)
    *out = RowsView{s->data, (long long)heads * n * d, (long long)n * d, d};
  for (long long st : {out->sb, out->sh, out->sn})
    if (st < 0 || st % 8 != 0) return RESTKV_ERR_INVALID_ARG;
  return RESTKV_OK;
}

}  // namespace restkv

using namespace restkv;

extern "C" {

size_t restkv_paged_page_bytes(const restkv_paged* cache) {
  PagedCache c;
  if (make_cache(cache, &c) != RESTKV_OK) return 0;
  return (size_t)c.Hkv * c.head_bytes;
}

static int device_sms() {
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) == cudaSuccess && cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) == cudaSuccess && sms > 0)
    return sms;
  (void)cudaGetLastError();
  return 148;
}

size_t restkv_paged_workspace_bytes(const restkv_paged* cache, int n_tokens) {
  PagedCache c;
  if (make_cache(cache, &c) != RESTKV_OK || check_tokens(c, n_tokens) != RESTKV_OK) return 0;
  c.n_tokens = n_tokens;
  return attend_bytes(c, cache->dtype == RESTKV_F32, device_sms());
}

restkv_status restkv_paged_append(restkv_handle* h, const restkv_paged* cache, int n_tokens, const restkv_rows* K_new,
                                  const restkv_rows* V_new, void* K_pages, void* V_pages, const int32_t* lengths,
                                  const int32_t* table, const int32_t* counts, const int32_t* positions,
                                  const restkv_rotation* rotation, const restkv_rows* Q, void* Q_out, restkv_stream stream) {
  if (!h || !K_pages || !V_pages || !lengths || !table) return RESTKV_ERR_INVALID_ARG;
  if (!aligned16(K_pages) || !aligned16(V_pages)) return RESTKV_ERR_INVALID_ARG;
  if ((Q == nullptr) != (Q_out == nullptr) || !aligned16(Q_out)) return RESTKV_ERR_INVALID_ARG;
  PagedCache c;
  restkv_status s = make_cache(cache, &c);
  if (s != RESTKV_OK) return s;
  if ((s = check_tokens(c, n_tokens)) != RESTKV_OK) return s;
  RowsView k, v, q{};
  if ((s = make_rows(K_new, c.Hkv, n_tokens, c.d, &k)) != RESTKV_OK) return s;
  if ((s = make_rows(V_new, c.Hkv, n_tokens, c.d, &v)) != RESTKV_OK) return s;
  if (Q && (s = make_rows(Q, c.Hq, n_tokens, c.d, &q)) != RESTKV_OK) return s;
  RotationView rot{};
  if (rotation) {
    if (!rotation->cos || !rotation->sin || !aligned16(rotation->cos) || !aligned16(rotation->sin)) return RESTKV_ERR_INVALID_ARG;
    if (rotation->n_positions < 1 || rotation->rotary_dim < 16 || rotation->rotary_dim % 16 != 0 || rotation->rotary_dim > c.d)
      return RESTKV_ERR_INVALID_ARG;
    if (rotation->interleaved != 0 && rotation->interleaved != 1) return RESTKV_ERR_INVALID_ARG;
    if (!positions && c.per_head) return RESTKV_ERR_INVALID_ARG;
    rot = RotationView{rotation->cos, rotation->sin, rotation->n_positions, rotation->rotary_dim / 2, rotation->interleaved};
  }
  c.lengths = lengths; c.table = table; c.counts = counts; c.n_tokens = n_tokens; c.dev_status = h->dev_status;
  Call call{h, (cudaStream_t)stream};
  RESTKV_LAUNCH(call, RESTKV_KERNEL_NONE,
                launch_paged_append(c, cache->dtype == RESTKV_F32, k, v, (uint8_t*)K_pages, (uint8_t*)V_pages, positions, rot, q, Q_out,
                                    h->sm_count, call.st), 1);
  return RESTKV_OK;
}

restkv_status restkv_paged_attend(restkv_handle* h, const restkv_paged* cache, int n_tokens, const restkv_rows* Q,
                                  const void* K_pages, const void* V_pages, const int32_t* lengths, const int32_t* table,
                                  const int32_t* counts, void* out, float* lse, void* workspace, size_t workspace_bytes,
                                  restkv_stream stream) {
  if (!h || !K_pages || !V_pages || !lengths || !table || !out) return RESTKV_ERR_INVALID_ARG;
  if (!aligned16(K_pages) || !aligned16(V_pages) || !aligned16(out)) return RESTKV_ERR_INVALID_ARG;
  PagedCache c;
  restkv_status s = make_cache(cache, &c);
  if (s != RESTKV_OK) return s;
  if ((s = check_tokens(c, n_tokens)) != RESTKV_OK) return s;
  RowsView q;
  if ((s = make_rows(Q, c.Hq, n_tokens, c.d, &q)) != RESTKV_OK) return s;
  c.lengths = lengths; c.table = table; c.counts = counts; c.n_tokens = n_tokens; c.dev_status = h->dev_status;
  c.K = (const uint8_t*)K_pages; c.V = (const uint8_t*)V_pages;
  if (!workspace || ((uintptr_t)workspace & 255u) != 0) return RESTKV_ERR_WORKSPACE;
  Call call{h, (cudaStream_t)stream};
  const bool f32 = cache->dtype == RESTKV_F32;
  if (workspace_bytes < attend_bytes(c, f32, h->sm_count)) return RESTKV_ERR_WORKSPACE;
  if (in_chunks(c, f32) && h->tc_state && h->kernel_path != 1) {
    RESTKV_LAUNCH(call, RESTKV_KERNEL_NONE,
                  launch_paged_chunk(c, q, out, lse, (float*)workspace, h->sm_count, h->wait_limit, call.st), 2);
    return RESTKV_OK;
  }
  if (on_tensor_pipe(c, f32) && h->tc_state && h->kernel_path != 1) {
    int launches = 0;
    RESTKV_LAUNCH(call, RESTKV_KERNEL_NONE,
                  launch_paged_mma(h->tc_state, c, q, out, lse, (float*)workspace, h->sm_count, h->paged_clusters,
                                   h->wait_limit, call.st, &launches), launches);
    return RESTKV_OK;
  }
  if (h->kernel_path >= 2) return RESTKV_ERR_UNSUPPORTED;   // the tensor cores are required
  const int splits = paged_simt_splits(c, h->sm_count);
  RESTKV_LAUNCH(call, RESTKV_KERNEL_NONE, launch_paged_simt(c, f32, q, out, lse, (float*)workspace, splits, call.st), splits == 1 ? 1 : 2);
  return RESTKV_OK;
}

restkv_status restkv_paged_read(restkv_handle* h, const restkv_paged* cache, const void* K_pages, const void* V_pages,
                                const int32_t* lengths, const int32_t* table, const int32_t* first, int n_rows, void* K_out,
                                void* V_out, restkv_stream stream) {
  if (!h || !K_pages || !V_pages || !lengths || !table || !K_out || !V_out || n_rows < 1) return RESTKV_ERR_INVALID_ARG;
  if (!aligned16(K_pages) || !aligned16(V_pages) || !aligned16(K_out) || !aligned16(V_out)) return RESTKV_ERR_INVALID_ARG;
  PagedCache c;
  const restkv_status s = make_cache(cache, &c);
  if (s != RESTKV_OK) return s;
  c.lengths = lengths; c.table = table; c.dev_status = h->dev_status;
  c.K = (const uint8_t*)K_pages; c.V = (const uint8_t*)V_pages;
  Call call{h, (cudaStream_t)stream};
  RESTKV_LAUNCH(call, RESTKV_KERNEL_NONE,
                launch_paged_read(c, cache->dtype == RESTKV_F32, first, n_rows, K_out, V_out, h->sm_count, call.st), 1);
  return RESTKV_OK;
}

restkv_status restkv_paged_reorder(restkv_handle* h, const restkv_paged* cache, int beams, const int32_t* parents, const int32_t* lengths,
                                   const int32_t* table, int32_t* table_out, int32_t* copies, int32_t* dropped, restkv_stream stream) {
  if (!h || !parents || !lengths || !table || !table_out || !copies || beams < 1) return RESTKV_ERR_INVALID_ARG;
  PagedCache c;
  const restkv_status s = make_cache(cache, &c);
  if (s != RESTKV_OK) return s;
  if (c.batch % beams != 0) return RESTKV_ERR_INVALID_ARG;
  if (c.per_head || beams > kBeamsMost) return RESTKV_ERR_UNSUPPORTED;
  // a table that is neither the other nor apart from it would be read where it has been written
  const size_t bytes = (size_t)c.batch * c.table_width * sizeof(int32_t);
  const uintptr_t from = (uintptr_t)table, to = (uintptr_t)table_out;
  if (from != to && from < to + bytes && to < from + bytes) return RESTKV_ERR_INVALID_ARG;
  if (!on_device(h)) return RESTKV_ERR_INVALID_ARG;
  c.lengths = lengths; c.table = table; c.dev_status = h->dev_status;
  Call call{h, (cudaStream_t)stream};
  RESTKV_LAUNCH(call, RESTKV_KERNEL_NONE, launch_paged_reorder(c, beams, parents, table, table_out, copies, dropped, call.st), 1);
  return RESTKV_OK;
}

restkv_status restkv_paged_copy(restkv_handle* h, const restkv_paged* cache, const int32_t* copies, int n_copies, void* K_pages, void* V_pages,
                                int n_layers, long long layer_bytes, restkv_stream stream) {
  if (!h || !copies || !K_pages || !V_pages || n_copies < 1 || n_layers < 1) return RESTKV_ERR_INVALID_ARG;
  if (!aligned16(K_pages) || !aligned16(V_pages)) return RESTKV_ERR_INVALID_ARG;
  PagedCache c;
  const restkv_status s = make_cache(cache, &c);
  if (s != RESTKV_OK) return s;
  const long long pool = (long long)c.n_pages * c.Hkv * c.head_bytes;
  if (layer_bytes == 0) layer_bytes = pool;
  if (layer_bytes < 0 || layer_bytes % 16 != 0 || (n_layers > 1 && layer_bytes < pool)) return RESTKV_ERR_INVALID_ARG;
  if ((long long)n_copies * n_layers > 0x7FFFFFFFll / (2 * c.Hkv)) return RESTKV_ERR_UNSUPPORTED;   // blocks of a grid
  if (!on_device(h)) return RESTKV_ERR_INVALID_ARG;
  c.dev_status = h->dev_status;
  Call call{h, (cudaStream_t)stream};
  RESTKV_LAUNCH(call, RESTKV_KERNEL_NONE,
                launch_paged_copy(c, copies, n_copies, n_layers, layer_bytes, (uint8_t*)K_pages, (uint8_t*)V_pages, call.st), 1);
  return RESTKV_OK;
}

}  // extern "C"
