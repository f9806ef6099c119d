// Cross attention in fp32 on the FMA pipe: single precision (whose products the tensor pipe would round), and bf16 with a head_dim or strides
// that the tensor-core kernels do not take.
//
// Split along the rows, kRows query rows share each row of K and V that is loaded, partial softmax per split, merged by log-sum-exp in
// a fixed order.  Bound by its FMAs for many rows and by the latency of two launches for few.
#include <math.h>

#include "cross.cuh"
#include "sm100_ptx.cuh"

namespace restkv {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kRows = 4, kAtOnce = 2;
constexpr int kMaxSplits = 64;

// grid (query rows / 4, splits, sources * Hkv); a single split writes the results itself.  A slot of `kLanes` threads takes a row of K and V, 8
// dims per thread; every slot keeps its own running (m, l, o) of the four query rows.
template <typename T, int kLanes>
__global__ void __launch_bounds__(kThreads) cross_simt_kernel(const CrossProblem c, float* __restrict__ part) {
  ptx::grid_dependency_wait();
  ptx::grid_dependency_launch();
  constexpr int kPerWarp = 32 / kLanes;
  const int splits = gridDim.y, split = blockIdx.y, bh = blockIdx.z, b = bh / c.Hkv, h = bh - b * c.Hkv;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, chunk = lane % kLanes;
  const bool has = chunk * 8 < c.d;
  const int R = (int)c.rows(), n = cross_length(c, b, h);
  float q[kRows][8], m[kRows], l[kRows], o[kRows][8];
  bool any = false;
#pragma unroll
  for (int k = 0; k < kRows; ++k) {
    const int rho = blockIdx.x * kRows + k;
    Pack8<T> p;
    p.zero();
    if (rho < R) {
      const CrossRow r = cross_row(c, b, rho);
      if (cross_live(c, r)) {
        any = true;
        if (has) p.load(cross_query<T>(c, r, h) + chunk * 8);
      }
    }
    p.get(q[k]);
    m[k] = -INFINITY;
    l[k] = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[k][e] = 0.f;
  }
  const long long blocks = any ? (n + 15) / 16 : 0;                     // whole runs of 16 rows per split
  const int r0 = (int)(blocks * split / splits) * 16, end = (int)(blocks * (split + 1) / splits) * 16, r1 = end < n ? end : n;
  const T* const K = reinterpret_cast<const T*>(c.K.data) + b * c.K.sb + h * c.K.sh + chunk * 8;
  const T* const V = reinterpret_cast<const T*>(c.V.data) + b * c.V.sb + h * c.V.sh + chunk * 8;
  // kAtOnce rows per slot together: their loads, sums and exponentials do not wait for one another, and the maximum is looked at once for all
  constexpr int kStep = kWarps * kPerWarp;
  for (int base = r0; base < r1; base += kAtOnce * kStep) {
    const int row0 = base + warp * kPerWarp + lane / kLanes;
    Pack8<T> kp[kAtOnce], vp[kAtOnce];
#pragma unroll
    for (int x = 0; x < kAtOnce; ++x) {
      kp[x].zero();
      vp[x].zero();
      if (has && row0 + x * kStep < r1) {
        kp[x].load(K + (row0 + x * kStep) * c.K.sn);
        vp[x].load(V + (row0 + x * kStep) * c.V.sn);
      }
    }
    float s[kRows][kAtOnce];
#pragma unroll
    for (int x = 0; x < kAtOnce; ++x) {
      float kf[8];
      kp[x].get(kf);
#pragma unroll
      for (int k = 0; k < kRows; ++k) {
        s[k][x] = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) s[k][x] = fmaf(q[k][e], kf[e], s[k][x]);
      }
    }
#pragma unroll
    for (int off = kLanes / 2; off > 0; off >>= 1)
#pragma unroll
      for (int k = 0; k < kRows; ++k)
#pragma unroll
        for (int x = 0; x < kAtOnce; ++x) s[k][x] += __shfl_xor_sync(0xffffffffu, s[k][x], off);
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
      float top = m[k];
#pragma unroll
      for (int x = 0; x < kAtOnce; ++x) {
        s[k][x] = row0 + x * kStep < r1 ? s[k][x] * c.scale : -INFINITY;
        top = fmaxf(top, s[k][x]);
      }
      const float of = top == -INFINITY ? 0.f : top;                       // only logits of -inf so far: they weigh nothing
      const float f = __expf(m[k] - of);                                   // m = -inf gives 0
      m[k] = top;
      l[k] *= f;
#pragma unroll
      for (int e = 0; e < 8; ++e) o[k][e] *= f;
#pragma unroll
      for (int x = 0; x < kAtOnce; ++x) {
        s[k][x] = __expf(s[k][x] - of);
        l[k] += s[k][x];
      }
    }
#pragma unroll
    for (int x = 0; x < kAtOnce; ++x) {
      float vf[8];
      vp[x].get(vf);
#pragma unroll
      for (int k = 0; k < kRows; ++k)
#pragma unroll
        for (int e = 0; e < 8; ++e) o[k][e] = fmaf(s[k][x], vf[e], o[k][e]);
    }
  }
  // merge: the slots of a warp by butterfly exchange, the warps through shared memory
#pragma unroll
  for (int off = kLanes; off < 32; off <<= 1) {
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
      const float mo = __shfl_xor_sync(0xffffffffu, m[k], off), lo = __shfl_xor_sync(0xffffffffu, l[k], off);
      const float mm = fmaxf(m[k], mo);
      const float sa = m[k] == -INFINITY ? 0.f : __expf(m[k] - mm), sb = mo == -INFINITY ? 0.f : __expf(mo - mm);
      l[k] = l[k] * sa + lo * sb;
#pragma unroll
      for (int e = 0; e < 8; ++e) o[k][e] = o[k][e] * sa + __shfl_xor_sync(0xffffffffu, o[k][e], off) * sb;
      m[k] = mm;
    }
  }
  __shared__ float w_ml[kWarps][kRows][2];
  __shared__ float w_o[kWarps][kRows][256];
  if (lane < kLanes && has) {
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
      if (chunk == 0) { w_ml[warp][k][0] = m[k]; w_ml[warp][k][1] = l[k]; }
#pragma unroll
      for (int e = 0; e < 8; ++e) w_o[warp][k][chunk * 8 + e] = o[k][e];
    }
  }
  __syncthreads();
  for (int e = threadIdx.x; e < kRows * c.d; e += kThreads) {
    const int k = e / c.d, dim = e - k * c.d, rho = blockIdx.x * kRows + k;
    if (rho >= R) continue;
    float mm = -INFINITY, acc = 0.f, ll = 0.f;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) mm = fmaxf(mm, w_ml[w][k][0]);
#pragma unroll
    for (int w = 0; w < kWarps; ++w) {
      const float mw = w_ml[w][k][0];
      const float f = mw == -INFINITY ? 0.f : __expf(mw - mm);
      acc = fmaf(w_o[w][k][dim], f, acc);
      ll = fmaf(w_ml[w][k][1], f, ll);
    }
    if (splits == 1) {
      const CrossRow r = cross_row(c, b, rho);
      const bool some = cross_some(c, r, ll);
      const long long row = cross_out_row(c, r, h);
      const float v = some ? acc / ll : 0.f;
      if constexpr (sizeof(T) == 4) reinterpret_cast<float*>(c.out)[row * c.d + dim] = v;
      else reinterpret_cast<__nv_bfloat16*>(c.out)[row * c.d + dim] = __float2bfloat16(v);
      if (c.lse && dim == 0) c.lse[row] = some ? mm + logf(ll) : -INFINITY;
    } else {
      float* to = part + (((long long)bh * R + rho) * splits + split) * (c.d + 2);
      to[2 + dim] = acc;
      if (dim == 0) { to[0] = mm; to[1] = ll; }
    }
  }
}

// grid (query rows, sources * Hkv): the splits of a query row.
template <typename T>
__global__ void cross_simt_combine_kernel(const CrossProblem c, int splits, const float* __restrict__ part) {
  ptx::grid_dependency_wait();
  ptx::grid_dependency_launch();
  const int R = (int)c.rows(), rho = blockIdx.x, bh = blockIdx.y, b = bh / c.Hkv, h = bh - b * c.Hkv;
  const CrossRow r = cross_row(c, b, rho);
  const float* from = part + ((long long)bh * R + rho) * splits * (c.d + 2);
  float mm = -INFINITY, ll = 0.f;
  for (int s = 0; s < splits; ++s) mm = fmaxf(mm, from[s * (c.d + 2)]);
  for (int s = 0; s < splits; ++s) {
    const float ms = from[s * (c.d + 2)];
    ll += ms == -INFINITY ? from[s * (c.d + 2) + 1] : from[s * (c.d + 2) + 1] * __expf(ms - mm);   // (0, or a sum that is no number)
  }
  const bool some = cross_some(c, r, ll);
  const long long row = cross_out_row(c, r, h);
  for (int k = threadIdx.x; k < c.d; k += blockDim.x) {
    float acc = 0.f;
    for (int s = 0; s < splits; ++s) {
      const float ms = from[s * (c.d + 2)];
      if (ms != -INFINITY) acc += from[s * (c.d + 2) + 2 + k] * __expf(ms - mm);
    }
    const float v = some ? acc / ll : 0.f;
    if constexpr (sizeof(T) == 4) reinterpret_cast<float*>(c.out)[row * c.d + k] = v;
    else reinterpret_cast<__nv_bfloat16*>(c.out)[row * c.d + k] = __float2bfloat16(v);
  }
  if (c.lse && threadIdx.x == 0) c.lse[row] = some ? mm + logf(ll) : -INFINITY;
}

template <typename T>
cudaError_t launch_t(const CrossProblem& c, float* part, int splits, cudaStream_t st) {
  void (*kernel)(CrossProblem, float*);
  switch (lanes_per_row(c.d)) {
    case 4: kernel = cross_simt_kernel<T, 4>; break;
    case 8: kernel = cross_simt_kernel<T, 8>; break;
    case 16: kernel = cross_simt_kernel<T, 16>; break;
    default: kernel = cross_simt_kernel<T, 32>;
  }
  const dim3 grid((unsigned int)((c.rows() + kRows - 1) / kRows), (unsigned int)splits, (unsigned int)(c.sources * c.Hkv));
  const cudaError_t e = launch_chained(kernel, grid, kThreads, 0, st, c, part);
  if (e != cudaSuccess || splits == 1) return e;
  return launch_chained(cross_simt_combine_kernel<T>, dim3((unsigned int)c.rows(), (unsigned int)(c.sources * c.Hkv)), (c.d + 31) / 32 * 32, 0, st, c, splits, part);
}

}  // namespace

int cross_simt_splits(const CrossProblem& c, int sm_count) {
  const long long units = (long long)c.sources * c.Hkv * ((c.rows() + kRows - 1) / kRows);
  long long splits = (2LL * sm_count + units - 1) / units;
  const long long by_rows = ((long long)c.n_rows + 63) / 64;
  if (splits > by_rows) splits = by_rows;
  if (splits > kMaxSplits) splits = kMaxSplits;
  return splits < 1 ? 1 : (int)splits;
}

// A bound of what the splits leave that never falls as the tokens grow: there are several only while four rows each make less than 2 units
// per SM, so that units * splits stays below 4 per SM.
size_t cross_simt_bytes(const CrossProblem& c, int sm_count) {
  const long long by_rows = ((long long)c.n_rows + 63) / 64, most = by_rows < kMaxSplits ? by_rows : kMaxSplits;
  const long long rows = (long long)c.sources * c.Hkv * c.rows(), bound = 4LL * 4 * sm_count;
  const long long slots = rows > bound / most ? bound : rows * most;   // (rows * most without leaving 64 bits)
  return (size_t)slots * (c.d + 2) * sizeof(float);
}

cudaError_t launch_cross_simt(const CrossProblem& c, bool f32, float* part, int splits, cudaStream_t st) {
  return f32 ? launch_t<float>(c, part, splits, st) : launch_t<__nv_bfloat16>(c, part, splits, st);
}

}  // namespace restkv
