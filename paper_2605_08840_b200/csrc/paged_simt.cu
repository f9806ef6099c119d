// Attention over the paged cache in fp32 on the FMA pipe: single precision (whose products the tensor pipe would round), and bf16
// with a head_dim that the tensor-core kernel has no instantiation for.
//
// Split along the rows, kSimtRows query rows (tokens x query heads of a KV head) share each cache row that is loaded, partial
// softmax per split, merged by log-sum-exp in a fixed order.  Bound by its FMAs in long caches and by the latency of two launches in short
// ones: 1024 rows of fp32, 8 heads of 64 over 2, 10.3 us.
#include <math.h>

#include "paged.cuh"
#include "sm100_ptx.cuh"

namespace restkv {

namespace {

constexpr int kSimtThreads = 256;
constexpr int kSimtRows = 4;
constexpr int kSimtMaxSplits = 64;

// grid (query rows / 4, splits, batch * Hkv); a single split writes the results itself.  A slot of `kLanes` threads takes a cache row, 8 dims
// per thread; every slot keeps its own running (m, l, o) of the four query rows.
template <typename T, bool kInt4, int kLanes>
__global__ void __launch_bounds__(kSimtThreads) paged_simt_kernel(const PagedCache c, const RowsView Q, float* __restrict__ part, T* __restrict__ out,
                                                                  float* __restrict__ lse) {
  ptx::grid_dependency_wait();
  constexpr int kPerWarp = 32 / kLanes, kWarps = kSimtThreads / 32;
  const int splits = gridDim.y, split = blockIdx.y, bh = blockIdx.z, b = bh / c.Hkv, h = bh - b * c.Hkv;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, chunk = lane % kLanes;
  const bool has = chunk * 8 < c.d;
  const int R = c.n_tokens * c.G, n = paged_length(c, b, h), count = paged_count(c, b);
  if (split == 0 && threadIdx.x == 0) check_length(c, b, h);
  int sees[kSimtRows];
  float q[kSimtRows][8], m[kSimtRows], l[kSimtRows], o[kSimtRows][8];
  int most = 0;
#pragma unroll
  for (int k = 0; k < kSimtRows; ++k) {
    const int rho = blockIdx.x * kSimtRows + k, i = rho / c.G, g = rho - i * c.G;
    sees[k] = rho < R && i < count ? n - (count - 1 - i) : 0;
    most = max(most, sees[k]);
    Pack8<T> p;
    p.zero();
    if (has && rho < R) p.load(reinterpret_cast<const T*>(Q.data) + b * Q.sb + (long long)(h * c.G + g) * Q.sh + i * Q.sn + chunk * 8);
    p.get(q[k]);
    m[k] = -INFINITY;
    l[k] = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[k][e] = 0.f;
  }
  // whole blocks of 16 rows per split
  const long long blocks = (most + kBlockRows - 1) / kBlockRows;
  const int r0 = (int)(blocks * split / splits) * kBlockRows, end = (int)(blocks * (split + 1) / splits) * kBlockRows;
  const int r1 = end < most ? end : most;
  for (int base = r0; base < r1; base += kWarps * kPerWarp) {
    const int row = base + warp * kPerWarp + lane / kLanes;
    bool in = row < r1;
    float kf[8], vf[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) kf[e] = vf[e] = 0.f;
    if (in) {
      const long long at = paged_block(c, b, h, row / kBlockRows);
      if (at < 0) {
        in = false;
        if (chunk == 0) atomicOr(c.dev_status, kDevBadIndex);
      } else if (has) {
        load_chunk<T, kInt4>(c, c.K + at, row % kBlockRows, chunk, true, kf);
        load_chunk<T, kInt4>(c, c.V + at, row % kBlockRows, chunk, false, vf);
      }
    }
#pragma unroll
    for (int k = 0; k < kSimtRows; ++k) {
      float s = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) s = fmaf(q[k][e], kf[e], s);
#pragma unroll
      for (int off = kLanes / 2; off > 0; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
      if (!in || row >= sees[k]) continue;
      s *= c.scale;
      if (c.softcap > 0.f) s = c.softcap * tanhf(s / c.softcap);
      if (s > m[k]) {
        const float f = __expf(m[k] - s);   // m = -inf gives 0
        l[k] *= f;
#pragma unroll
        for (int e = 0; e < 8; ++e) o[k][e] *= f;
        m[k] = s;
      }
      const float p = m[k] == -INFINITY ? 0.f : __expf(s - m[k]);   // only logits of -inf so far: they weigh nothing
      l[k] += p;
#pragma unroll
      for (int e = 0; e < 8; ++e) o[k][e] = fmaf(p, vf[e], o[k][e]);
    }
  }
  // merge: the slots of a warp by butterfly exchange, the warps through shared memory
#pragma unroll
  for (int off = kLanes; off < 32; off <<= 1) {
#pragma unroll
    for (int k = 0; k < kSimtRows; ++k) {
      const float mo = __shfl_xor_sync(0xffffffffu, m[k], off), lo = __shfl_xor_sync(0xffffffffu, l[k], off);
      const float mm = fmaxf(m[k], mo);
      const float sa = m[k] == -INFINITY ? 0.f : __expf(m[k] - mm), sb = mo == -INFINITY ? 0.f : __expf(mo - mm);
      l[k] = l[k] * sa + lo * sb;
#pragma unroll
      for (int e = 0; e < 8; ++e) o[k][e] = o[k][e] * sa + __shfl_xor_sync(0xffffffffu, o[k][e], off) * sb;
      m[k] = mm;
    }
  }
  __shared__ float w_ml[kWarps][kSimtRows][2];
  __shared__ float w_o[kWarps][kSimtRows][256];
  if (lane < kLanes && has) {
#pragma unroll
    for (int k = 0; k < kSimtRows; ++k) {
      if (chunk == 0) { w_ml[warp][k][0] = m[k]; w_ml[warp][k][1] = l[k]; }
#pragma unroll
      for (int e = 0; e < 8; ++e) w_o[warp][k][chunk * 8 + e] = o[k][e];
    }
  }
  __syncthreads();
  for (int e = threadIdx.x; e < kSimtRows * c.d; e += kSimtThreads) {
    const int k = e / c.d, dim = e - k * c.d, rho = blockIdx.x * kSimtRows + k;
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
      const int i = rho / c.G, g = rho - i * c.G;
      const long long row = ((long long)b * c.Hq + h * c.G + g) * c.n_tokens + i;
      const float v = ll > 0.f ? acc / ll : 0.f;
      if constexpr (sizeof(T) == 4) out[row * c.d + dim] = v;
      else out[row * c.d + dim] = __float2bfloat16(v);
      if (lse && dim == 0) lse[row] = ll > 0.f ? mm + logf(ll) : -INFINITY;
    } else {
      float* to = part + (((long long)bh * R + rho) * splits + split) * (c.d + 2);
      to[2 + dim] = acc;
      if (dim == 0) { to[0] = mm; to[1] = ll; }
    }
  }
}

// grid (query rows, batch * Hkv): the splits of a query row.
template <typename T>
__global__ void paged_simt_combine_kernel(const PagedCache c, int splits, const float* __restrict__ part, T* __restrict__ out,
                                          float* __restrict__ lse) {
  ptx::grid_dependency_wait();
  const int R = c.n_tokens * c.G, rho = blockIdx.x, bh = blockIdx.y, b = bh / c.Hkv, h = bh - b * c.Hkv;
  const int i = rho / c.G, g = rho - i * c.G;
  const float* from = part + ((long long)bh * R + rho) * splits * (c.d + 2);
  float mm = -INFINITY, ll = 0.f;
  for (int s = 0; s < splits; ++s) mm = fmaxf(mm, from[s * (c.d + 2)]);
  for (int s = 0; s < splits; ++s) {
    const float ms = from[s * (c.d + 2)];
    if (ms != -INFINITY) ll += from[s * (c.d + 2) + 1] * __expf(ms - mm);
  }
  const long long row = ((long long)b * c.Hq + h * c.G + g) * c.n_tokens + i;
  for (int k = threadIdx.x; k < c.d; k += blockDim.x) {
    float acc = 0.f;
    for (int s = 0; s < splits; ++s) {
      const float ms = from[s * (c.d + 2)];
      if (ms != -INFINITY) acc += from[s * (c.d + 2) + 2 + k] * __expf(ms - mm);
    }
    const float v = ll > 0.f ? acc / ll : 0.f;
    if constexpr (sizeof(T) == 4) out[row * c.d + k] = v;
    else out[row * c.d + k] = __float2bfloat16(v);
  }
  if (lse && threadIdx.x == 0) lse[row] = ll > 0.f ? mm + logf(ll) : -INFINITY;
}

template <typename T, bool kInt4>
void (*pick_simt(int lanes))(PagedCache, RowsView, float*, T*, float*) {
  switch (lanes) {
    case 4: return paged_simt_kernel<T, kInt4, 4>;
    case 8: return paged_simt_kernel<T, kInt4, 8>;
    case 16: return paged_simt_kernel<T, kInt4, 16>;
    default: return paged_simt_kernel<T, kInt4, 32>;
  }
}

template <typename T>
cudaError_t launch_t(const PagedCache& c, const RowsView& Q, T* out, float* lse, float* part, int splits, cudaStream_t st) {
  const int R = c.n_tokens * c.G;
  const auto kernel = c.format == RESTKV_PAGES_INT4 ? pick_simt<T, true>(lanes_per_row(c.d)) : pick_simt<T, false>(lanes_per_row(c.d));
  const dim3 grid((unsigned int)((R + kSimtRows - 1) / kSimtRows), (unsigned int)splits, (unsigned int)(c.batch * c.Hkv));
  const cudaError_t e = launch_chained(kernel, grid, kSimtThreads, 0, st, c, Q, part, out, lse);
  if (e != cudaSuccess || splits == 1) return e;
  return launch_chained(paged_simt_combine_kernel<T>, dim3((unsigned int)R, (unsigned int)(c.batch * c.Hkv)), (c.d + 31) / 32 * 32, 0, st, c,
                        splits, part, out, lse);
}

}  // namespace

int paged_simt_splits(const PagedCache& c, int sm_count) {
  const long long units = (long long)c.batch * c.Hkv * ((c.n_tokens * (long long)c.G + kSimtRows - 1) / kSimtRows);
  long long splits = (2LL * sm_count + units - 1) / units;
  const long long by_rows = (c.capacity() + 63) / 64;
  if (splits > by_rows) splits = by_rows;
  if (splits > kSimtMaxSplits) splits = kSimtMaxSplits;
  return splits < 1 ? 1 : (int)splits;
}

// A bound of what the splits leave that never falls as the tokens grow: there are several only while four rows each make less than 2 units
// per SM, so that units * splits stays below 4 per SM.
size_t paged_simt_bytes(const PagedCache& c, int sm_count) {
  const long long by_rows = (c.capacity() + 63) / 64, most = by_rows < kSimtMaxSplits ? by_rows : kSimtMaxSplits;
  const long long rows = (long long)c.batch * c.Hq * c.n_tokens * most, bound = 4LL * 4 * sm_count;
  return (size_t)(rows < bound ? rows : bound) * (c.d + 2) * sizeof(float);
}

cudaError_t launch_paged_simt(const PagedCache& c, bool f32, const RowsView& Q, void* out, float* lse, float* part, int splits, cudaStream_t st) {
  return f32 ? launch_t(c, Q, (float*)out, lse, part, splits, st) : launch_t(c, Q, (__nv_bfloat16*)out, lse, part, splits, st);
}

}  // namespace restkv
