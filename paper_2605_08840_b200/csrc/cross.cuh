// Cross attention: its description as the kernels get it.
#pragma once

#include "paged.cuh"

namespace restkv {

struct CrossProblem {
  int sources, beams, Hq, Hkv, G, d;
  int n_rows, per_head;       // lengths [sources, Hkv] instead of [sources]
  int n_tokens;
  float scale;
  const int *lengths, *counts;   // null: n_rows, n_tokens
  RowsView Q, K, V;
  void* out;
  float* lse;                 // or null

  __host__ __device__ long long rows() const { return (long long)beams * n_tokens * G; }   // query rows of a KV head
};

// Query row rho of a KV head: sequence, token, head of the group in turn, the last running fastest.
struct CrossRow {
  int seq, i, g;
};
__device__ __forceinline__ CrossRow cross_row(const CrossProblem& c, int source, int rho) {
  const int x = rho / c.G, beam = x / c.n_tokens;
  return CrossRow{source * c.beams + beam, x - beam * c.n_tokens, rho - x * c.G};
}
__device__ __forceinline__ bool cross_live(const CrossProblem& c, const CrossRow& r) { return !c.counts || r.i < c.counts[r.seq]; }
// Whether a query row has a result: rows of K that weigh something, or logits that are no numbers, which make the sum of the weights none (a logit of
// +inf does, too: its weight is 2^(inf - inf)) and with it the row's outputs and log-sum-exp.
__device__ __forceinline__ bool cross_some(const CrossProblem& c, const CrossRow& r, float l) { return l != 0.f && cross_live(c, r); }
__device__ __forceinline__ int cross_length(const CrossProblem& c, int source, int h) {
  if (!c.lengths) return c.n_rows;
  const int n = c.lengths[c.per_head ? source * c.Hkv + h : source];
  return n < 0 ? 0 : n < c.n_rows ? n : c.n_rows;
}
template <typename T> __device__ __forceinline__ const T* cross_query(const CrossProblem& c, const CrossRow& r, int h) {
  return reinterpret_cast<const T*>(c.Q.data) + r.seq * c.Q.sb + (long long)(h * c.G + r.g) * c.Q.sh + r.i * c.Q.sn;
}
__device__ __forceinline__ long long cross_out_row(const CrossProblem& c, const CrossRow& r, int h) {
  return ((long long)r.seq * c.Hq + h * c.G + r.g) * c.n_tokens + r.i;
}

// fp32 SIMT: every dtype and head_dim
int cross_simt_splits(const CrossProblem& c, int sm_count);
size_t cross_simt_bytes(const CrossProblem& c, int sm_count);
cudaError_t launch_cross_simt(const CrossProblem& c, bool f32, float* part, int splits, cudaStream_t st);
// bf16 with head_dim 64 or 128 on the warp-level tensor instructions, up to 32 query rows per pass over K and V
cudaError_t cross_few_init();
bool cross_few_supported(const CrossProblem& c);
size_t cross_few_bytes(const CrossProblem& c, int sm_count);
double cross_few_us(const CrossProblem& c, const int* clusters_of);   // about how long it would take
cudaError_t launch_cross_few(void* state, const CrossProblem& c, float* part, int sm_count, const int* clusters_of, long long wait_limit, unsigned int* dev_status,
                             cudaStream_t st, int* launches);
// the same on tcgen05, 256 query rows per pass: from kManyRows of them on, where it takes less time
constexpr int kManyRows = 33;
cudaError_t cross_many_init();
bool cross_many_supported(const CrossProblem& c);
size_t cross_many_bytes(const CrossProblem& c, int sm_count);
double cross_many_us(const CrossProblem& c, int sm_count);
cudaError_t launch_cross_many(void* state, const CrossProblem& c, float* part, int sm_count, long long wait_limit, unsigned int* dev_status, cudaStream_t st);

}  // namespace restkv
