// The handle behind the C ABI and what every entry point shares: alignment checks, the launch bookkeeping.
#pragma once

#include <atomic>

#include "restkv_common.cuh"

struct restkv_handle {
  int device;
  int sm_count;
  unsigned int* dev_status;   // device block of kDevWords: word 0 = sticky status bits, then the sets of barrier counters
  std::atomic<unsigned int> counter_turn[2];   // launches so far that took a set: called, recorded into graphs
  void* tc_state;
  bool cross_few, cross_many; // whether these kernels of the cross attention can run (tc_state says so for all others on the tensor cores)
  int select_clusters[4];     // clusters of 1, 2, 4, 8 CTAs of the select kernel that the device holds at once
  int decode_clusters[5];     // clusters of 1, 2, 4, 8, 16 CTAs of the decode kernel that the device holds at once
  int paged_clusters[2][5];   // the same of the paged attention kernels with one and with two CTAs per SM
  long long launches;
  int last_cuda_error;
  int kernel_path;            // 0 auto, 1 SIMT, 2 tensor core required, 3 tensor core in its head-sequential form
  bool fused_select;          // restkv_evict chains the launch that pools, selects and gathers to the score kernel
  bool last_evict_fused;      // whether the last restkv_evict did
  long long wait_limit;       // SM clocks a device-side wait may last
  restkv_variant variant;     // ablation variant of the score calls (all 0: the method as printed)
  const void* proj_factor;    // output-projection factor of the score calls (null: identity), caller-owned
  int proj_heads, proj_dim;   // the shape it was prepared for
  cudaEvent_t prof_start[7], prof_stop[7];   // per restkv_kernel_id, null = not timed
};

namespace restkv {

inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }
// Whether the handle's device is the current one, on which a launch would go.
inline bool on_device(const restkv_handle* h) {
  int dev = -1;
  if (cudaGetDevice(&dev) == cudaSuccess) return dev == h->device;
  (void)cudaGetLastError();
  return false;
}
inline bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }

struct Call {
  restkv_handle* h;
  cudaStream_t st;
  // the barrier counters of the next persistent launch
  unsigned int* counters() {
    cudaStreamCaptureStatus capture = cudaStreamCaptureStatusNone;
    if (cudaStreamIsCapturing(st, &capture) != cudaSuccess) {
      (void)cudaGetLastError();   // the legacy stream beside a capture in another one: the launch itself will say so
      capture = cudaStreamCaptureStatusNone;
    }
    const unsigned int recorded = capture == cudaStreamCaptureStatusNone ? 0u : 1u;
    const unsigned int turn = h->counter_turn[recorded].fetch_add(1u, std::memory_order_relaxed) % kCounterSets;
    return h->dev_status + kDevStatusWords + (recorded * kCounterSets + turn) * kDevCounterWords;
  }
  restkv_status fail(cudaError_t e) {
    h->last_cuda_error = (int)e;
    return RESTKV_ERR_CUDA;
  }
};

#define RESTKV_LAUNCH(call, id, expr, count)                                                    \
  do {                                                                                          \
    const bool prof__ = (call).h->prof_start[(id)] != nullptr;                                  \
    if (prof__) cudaEventRecord((call).h->prof_start[(id)], (call).st);                         \
    cudaError_t e__ = (expr);                                                                   \
    if (e__ != cudaSuccess) return (call).fail(e__);                                            \
    if (prof__) cudaEventRecord((call).h->prof_stop[(id)], (call).st);                          \
    (call).h->launches += (count);                                                              \
  } while (0)

}  // namespace restkv
