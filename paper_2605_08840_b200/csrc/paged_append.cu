// Rows into and out of the paged cache.
#include "paged.cuh"
#include "sm100_ptx.cuh"

namespace restkv {

namespace {

constexpr int kRowThreads = 128;

// 8 dims of a row from (and to) their place in a block of 16 rows; `chunk` = dim / 8.
template <typename T, bool kInt4>
__device__ __forceinline__ void store_chunk(const PagedCache& c, uint8_t* block, int r, int chunk, bool is_key, const float* x, float lo,
                                            float step) {
  if constexpr (!kInt4) {
    Pack8<T>::store(reinterpret_cast<T*>(block + (long long)r * c.row_bytes) + chunk * 8, x);
  } else {
    unsigned int w = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) w |= int4_code(x[i], lo, step) << (4 * i);
    const int m = chunk >> 2, q = chunk & 3, words = c.d >> 5;
    uint8_t* row = block + r * c.row_bytes;
    if (is_key) {
      reinterpret_cast<unsigned int*>(row)[q * words + m] = w;
    } else {
      unsigned short* v = reinterpret_cast<unsigned short*>(row);
      v[2 * q * words + m] = (unsigned short)(w & 0xFFFFu);
      v[(2 * q + 1) * words + m] = (unsigned short)(w >> 16);
    }
    if ((chunk * 8) % c.group == 0) {
      unsigned short* p = reinterpret_cast<unsigned short*>(block + int4_params(c.d, chunk * 8 / c.group, r));
      p[0] = (unsigned short)(__float_as_uint(step) >> 16);
      p[4] = (unsigned short)(__float_as_uint(lo) >> 16);
    }
  }
}

// grid (batch * n_tokens, y); a slot of `lanes` threads takes a row of one head: heads slot, slot + slots, ... of Q, K and V, so that
// the token's cosines and sines are read once and stay in registers.  What bounds it: HBM (every row is read and written once), or
// for one token the latency of lengths -> table -> row.
template <typename T, bool kInt4>
__global__ void __launch_bounds__(kRowThreads) paged_append_kernel(const PagedCache c, const RowsView Kn, const RowsView Vn, uint8_t* K_pages,
                                                                   uint8_t* V_pages, const int* __restrict__ positions, const RotationView rot,
                                                                   const RowsView Q, T* Q_out, int lanes) {
  ptx::grid_dependency_wait();
  const int b = blockIdx.x / c.n_tokens, i = blockIdx.x - b * c.n_tokens;
  const int slots = kRowThreads / lanes, slot = threadIdx.x / lanes, chunk = threadIdx.x % lanes;
  const bool has = chunk * 8 < c.d;
  const int count = paged_count(c, b);
  const bool there = i < count;
  const int n_q = Q.data ? c.Hq : 0;
  const int heads = n_q + 2 * c.Hkv;
  float cs[8], sn[8];
  bool turns = false, placed = true;
  if (there && rot.cos) {
    const int p = positions ? positions[(long long)b * c.n_tokens + i] : c.lengths[b] - count + i;
    placed = (unsigned int)p < (unsigned int)rot.n_positions;
    if (!placed && threadIdx.x == 0) atomicOr(c.dev_status, kDevBadIndex);
    turns = placed && chunk * 8 < 2 * rot.half;
    if (turns) {
      // in halves 8 angles from the chunk's place in its half on, interleaved 4 of them twice
      const long long at = (long long)p * rot.half + (rot.interleaved ? chunk * 4 : chunk * 8 % rot.half);
      float4 v[4];
      v[0] = *reinterpret_cast<const float4*>(rot.cos + at);
      v[2] = *reinterpret_cast<const float4*>(rot.sin + at);
      if (!rot.interleaved) {
        v[1] = *reinterpret_cast<const float4*>(rot.cos + at + 4);
        v[3] = *reinterpret_cast<const float4*>(rot.sin + at + 4);
        const float* f = &v[0].x;
#pragma unroll
        for (int e = 0; e < 8; ++e) { cs[e] = f[e]; sn[e] = f[8 + e]; }
      } else {
        const float* f = &v[0].x;
#pragma unroll
        for (int e = 0; e < 8; ++e) { cs[e] = f[e / 2]; sn[e] = f[8 + e / 2]; }
      }
    }
  }
  for (int head = blockIdx.y * slots + slot; head - slot < heads; head += gridDim.y * slots) {   // whole warps stay: they exchange halves
    const bool mine = head < heads && has;
    const int kind = head < n_q ? 0 : head < n_q + c.Hkv ? 1 : 2;   // Q, K, V
    const int h = kind == 0 ? head : kind == 1 ? head - n_q : head - n_q - c.Hkv;
    const RowsView& src = kind == 0 ? Q : kind == 1 ? Kn : Vn;
    Pack8<T> raw;
    raw.zero();
    if (mine && there) raw.load(reinterpret_cast<const T*>(src.data) + b * src.sb + h * src.sh + i * src.sn + chunk * 8);
    float x[8];
    raw.get(x);
    if (rot.cos) {
      // every lane takes part in the exchange: a row of V may share the warp
      float other[8];
      const int half_chunks = rot.half >> 3;
      const int partner = (threadIdx.x & 31) + (rot.interleaved || !turns ? 0 : chunk < half_chunks ? half_chunks : -half_chunks);
#pragma unroll
      for (int e = 0; e < 8; ++e) other[e] = __shfl_sync(0xffffffffu, x[e], partner & 31);
      if (turns && kind != 2) {
        if (rot.interleaved) {
#pragma unroll
          for (int e = 0; e < 8; e += 2) {
            const float a = x[e], bb = x[e + 1];
            x[e] = __fsub_rn(__fmul_rn(a, cs[e]), __fmul_rn(bb, sn[e]));
            x[e + 1] = __fadd_rn(__fmul_rn(bb, cs[e]), __fmul_rn(a, sn[e]));
          }
        } else if (chunk < half_chunks) {
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = __fsub_rn(__fmul_rn(x[e], cs[e]), __fmul_rn(other[e], sn[e]));
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = __fadd_rn(__fmul_rn(x[e], cs[e]), __fmul_rn(other[e], sn[e]));
        }
      }
    }
    float lo = 0.f, step = 0.f;
    if constexpr (kInt4) {
      if (kind != 0) {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = int4_input(x[e]);
      }
      float hi = x[0];
      lo = x[0];
#pragma unroll
      for (int e = 1; e < 8; ++e) { lo = fminf(lo, x[e]); hi = fmaxf(hi, x[e]); }
      for (int off = 1; off < c.group / 8; off <<= 1) {
        lo = fminf(lo, __shfl_xor_sync(0xffffffffu, lo, off));
        hi = fmaxf(hi, __shfl_xor_sync(0xffffffffu, hi, off));
      }
      lo = bf16_below(lo);
      step = bf16_above(__fdiv_rn(hi - lo, 15.f));
    }
    if (!mine) continue;
    if (kind == 0) {
      if (!there || placed) Pack8<T>::store(Q_out + (((long long)b * c.Hq + h) * c.n_tokens + i) * c.d + chunk * 8, x);
      continue;
    }
    if (!there || !placed) continue;
    const long long row = (long long)c.lengths[c.per_head ? b * c.Hkv + h : b] - count + i;
    long long at = -1;
    if (row >= 0 && row < c.capacity()) at = paged_block(c, b, h, (int)(row / kBlockRows));
    if (at < 0) {
      if (chunk == 0) atomicOr(c.dev_status, kDevBadIndex);
      continue;
    }
    store_chunk<T, kInt4>(c, (kind == 1 ? K_pages : V_pages) + at, (int)(row % kBlockRows), chunk, kind == 1, x, lo, step);
  }
}

// grid (rows / slots, batch * Hkv, 2): K and V rows first .. first + n_rows of every head, a slot of `lanes` threads per row.
template <typename T, bool kInt4>
__global__ void __launch_bounds__(kRowThreads) paged_read_kernel(const PagedCache c, const int* __restrict__ first, int n_rows, T* K_out,
                                                                 T* V_out, int lanes) {
  ptx::grid_dependency_wait();
  const int bh = blockIdx.y, b = bh / c.Hkv, h = bh - b * c.Hkv;
  const bool is_key = blockIdx.z == 0;
  const int chunk = threadIdx.x % lanes;
  const int i = blockIdx.x * (kRowThreads / lanes) + threadIdx.x / lanes;
  if (i >= n_rows || chunk * 8 >= c.d) return;
  if (i == 0 && chunk == 0) check_length(c, b, h);
  const long long row = (long long)(first ? first[c.per_head ? bh : b] : 0) + i;
  float x[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) x[e] = 0.f;
  if (row >= 0 && row < paged_length(c, b, h)) {
    const long long at = paged_block(c, b, h, (int)(row / kBlockRows));
    if (at < 0) {
      if (chunk == 0) atomicOr(c.dev_status, kDevBadIndex);
    } else {
      const uint8_t* block = (is_key ? c.K : c.V) + at;
      const int r = (int)(row % kBlockRows);
      if constexpr (!kInt4) {
        Pack8<T> p;
        p.load(reinterpret_cast<const T*>(block + (long long)r * c.row_bytes) + chunk * 8);
        p.get(x);
      } else {
        const int m = chunk >> 2, q = chunk & 3, words = c.d >> 5;
        const uint8_t* codes = block + r * c.row_bytes;
        unsigned int w;
        if (is_key) {
          w = reinterpret_cast<const unsigned int*>(codes)[q * words + m];
        } else {
          const unsigned short* v = reinterpret_cast<const unsigned short*>(codes);
          w = v[2 * q * words + m] | (unsigned int)v[(2 * q + 1) * words + m] << 16;
        }
        const unsigned short* p = reinterpret_cast<const unsigned short*>(block + int4_params(c.d, chunk * 8 / c.group, r));
        const float step = __uint_as_float((unsigned int)p[0] << 16), lo = __uint_as_float((unsigned int)p[4] << 16);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = fmaf(step, (float)(w >> (4 * e) & 15u), lo);   // step * code is exact: one rounding
      }
    }
  }
  Pack8<T>::store((is_key ? K_out : V_out) + ((long long)bh * n_rows + i) * c.d + chunk * 8, x);
}

int lanes_per_row(int d) {
  int lanes = 4;
  while (lanes * 8 < d) lanes *= 2;
  return lanes;
}

}  // namespace

cudaError_t launch_paged_append(const PagedCache& c, bool f32, const RowsView& Kn, const RowsView& Vn, uint8_t* K_pages, uint8_t* V_pages,
                                const int* positions, const RotationView& rot, const RowsView& Q, void* Q_out, int sm_count, cudaStream_t st) {
  const int lanes = lanes_per_row(c.d), slots = kRowThreads / lanes;
  const long long tokens = (long long)c.batch * c.n_tokens;
  const int heads = (Q.data ? c.Hq : 0) + 2 * c.Hkv;
  // one block per token reads the token's angles once; with few tokens the heads go to blocks of their own until there are 4 per SM
  long long y = (4 * sm_count + tokens - 1) / tokens;
  const int most = (heads + slots - 1) / slots;
  if (y > most) y = most;
  const dim3 grid((unsigned int)tokens, (unsigned int)y);
  const bool int4 = c.format == RESTKV_PAGES_INT4;
  if (f32)
    return launch_chained(int4 ? paged_append_kernel<float, true> : paged_append_kernel<float, false>, grid, kRowThreads, 0, st, c, Kn, Vn,
                          K_pages, V_pages, positions, rot, Q, (float*)Q_out, lanes);
  return launch_chained(int4 ? paged_append_kernel<__nv_bfloat16, true> : paged_append_kernel<__nv_bfloat16, false>, grid, kRowThreads, 0, st,
                        c, Kn, Vn, K_pages, V_pages, positions, rot, Q, (__nv_bfloat16*)Q_out, lanes);
}

cudaError_t launch_paged_read(const PagedCache& c, bool f32, const int* first, int n_rows, void* K_out, void* V_out, cudaStream_t st) {
  const int lanes = lanes_per_row(c.d), slots = kRowThreads / lanes;
  const dim3 grid((unsigned int)((n_rows + slots - 1) / slots), (unsigned int)(c.batch * c.Hkv), 2);
  const bool int4 = c.format == RESTKV_PAGES_INT4;
  if (f32)
    return launch_chained(int4 ? paged_read_kernel<float, true> : paged_read_kernel<float, false>, grid, kRowThreads, 0, st, c, first, n_rows,
                          (float*)K_out, (float*)V_out, lanes);
  return launch_chained(int4 ? paged_read_kernel<__nv_bfloat16, true> : paged_read_kernel<__nv_bfloat16, false>, grid, kRowThreads, 0, st, c,
                        first, n_rows, (__nv_bfloat16*)K_out, (__nv_bfloat16*)V_out, lanes);
}

}  // namespace restkv
