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
// the token's cosines and sines are read once and stay in registers, kUnroll rows at a time, all of them on their way before the first
// is needed.  What bounds it: HBM (every row is read and written once), or for one token the latency of lengths -> table -> row.
template <typename T, bool kInt4, int kUnroll>
__global__ void __launch_bounds__(kRowThreads) paged_append_kernel(const PagedCache c, const RowsView Kn, const RowsView Vn, uint8_t* K_pages,
                                                                   uint8_t* V_pages, const int* __restrict__ positions, const RotationView rot,
                                                                   const RowsView Q, T* Q_out, int lanes) {
  ptx::grid_dependency_wait();
  ptx::grid_dependency_launch();
  const int b = blockIdx.x / c.n_tokens, i = blockIdx.x - b * c.n_tokens;
  const int slots = kRowThreads / lanes, slot = threadIdx.x / lanes, chunk = threadIdx.x % lanes;
  const bool has = chunk * 8 < c.d;
  const int n_q = Q.data ? c.Hq : 0, heads = n_q + 2 * c.Hkv, stride = gridDim.y * slots;
  const T* const q_row = reinterpret_cast<const T*>(Q.data) + b * Q.sb + i * Q.sn + chunk * 8;
  const T* const k_row = reinterpret_cast<const T*>(Kn.data) + b * Kn.sb + i * Kn.sn + chunk * 8;
  const T* const v_row = reinterpret_cast<const T*>(Vn.data) + b * Vn.sb + i * Vn.sn + chunk * 8;
  auto row_of = [&](int head) {
    return head < n_q ? q_row + head * Q.sh : head < n_q + c.Hkv ? k_row + (head - n_q) * Kn.sh : v_row + (head - n_q - c.Hkv) * Vn.sh;
  };
  // whole warps stay in the loop: its rounds go by the block's first head.  (Rows past a count are loaded, too: they are the caller's.)
  int head = blockIdx.y * slots + slot;
  Pack8<T> raw[kUnroll];
  auto load = [&]() {
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      raw[u].zero();
      if (has && head + u * stride < heads) raw[u].load(row_of(head + u * stride));
    }
  };
  load();
  const int count = paged_count(c, b);
  const bool there = i < count;
  // where the token goes; with lengths per head that is each head's own matter
  const int per_page = c.page_rows / kBlockRows;
  int page = -1;
  long long row = 0;
  auto find = [&](int h) {
    row = (long long)c.lengths[c.per_head ? b * c.Hkv + h : b] - count + i;
    page = row >= 0 && row < c.capacity() ? c.table[(long long)b * c.table_width + (int)row / c.page_rows] : -1;
  };
  if (there && !c.per_head) find(0);
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
      const float4 c0 = *reinterpret_cast<const float4*>(rot.cos + at), s0 = *reinterpret_cast<const float4*>(rot.sin + at);
      if (rot.interleaved) {
        cs[0] = cs[1] = c0.x; cs[2] = cs[3] = c0.y; cs[4] = cs[5] = c0.z; cs[6] = cs[7] = c0.w;
        sn[0] = sn[1] = s0.x; sn[2] = sn[3] = s0.y; sn[4] = sn[5] = s0.z; sn[6] = sn[7] = s0.w;
      } else {
        const float4 c1 = *reinterpret_cast<const float4*>(rot.cos + at + 4), s1 = *reinterpret_cast<const float4*>(rot.sin + at + 4);
        cs[0] = c0.x; cs[1] = c0.y; cs[2] = c0.z; cs[3] = c0.w; cs[4] = c1.x; cs[5] = c1.y; cs[6] = c1.z; cs[7] = c1.w;
        sn[0] = s0.x; sn[1] = s0.y; sn[2] = s0.z; sn[3] = s0.w; sn[4] = s1.x; sn[5] = s1.y; sn[6] = s1.z; sn[7] = s1.w;
      }
    }
  }
  const int half_chunks = rot.half >> 3;
  const int partner = ((threadIdx.x & 31) + (rot.interleaved || !turns ? 0 : chunk < half_chunks ? half_chunks : -half_chunks)) & 31;
  for (;;) {
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) {
      const int hd = head + u * stride;
      if (hd - slot >= heads) break;
      const bool mine = hd < heads && has;
      const int kind = hd < n_q ? 0 : hd < n_q + c.Hkv ? 1 : 2;   // Q, K, V
      const int h = kind == 0 ? hd : kind == 1 ? hd - n_q : hd - n_q - c.Hkv;
      float x[8];
      raw[u].get(x);
      if (rot.cos) {
        // every lane takes part in the exchange: a row of V may share the warp
        float other[8];
        raw[u].exchange(partner, other);
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
        if (__any_sync(0xffffffffu, kind != 0)) {
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
      }
      if (!mine) continue;
      if (kind == 0) {
        if (!there) {
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = 0.f;
        }
        if (placed) Pack8<T>::store(Q_out + (((long long)b * c.Hq + h) * c.n_tokens + i) * c.d + chunk * 8, x);
        continue;
      }
      if (!there || !placed) continue;
      if (c.per_head) find(h);
      if ((unsigned int)page >= (unsigned int)c.n_pages) {
        if (chunk == 0) atomicOr(c.dev_status, kDevBadIndex);
        continue;
      }
      const long long block = ((long long)page * c.Hkv + h) * per_page + (int)row % c.page_rows / kBlockRows;
      store_chunk<T, kInt4>(c, (kind == 1 ? K_pages : V_pages) + block * c.block_bytes, (int)row % kBlockRows, chunk, kind == 1, x, lo, step);
    }
    head += kUnroll * stride;
    if (head - slot >= heads) return;
    load();
  }
}

// grid (blocks of 16 rows, batch * Hkv / warps): a warp takes 16 rows of K or V of a head, so that the page is looked up once for them
// and all of their loads are on their way together.  Rows first .. first + n_rows of every head.
template <typename T, bool kInt4, int kLanes>
__global__ void __launch_bounds__(kRowThreads) paged_read_kernel(const PagedCache c, const int* __restrict__ first, int n_rows, T* K_out,
                                                                 T* V_out) {
  ptx::grid_dependency_wait();
  ptx::grid_dependency_launch();
  const int lane = threadIdx.x & 31, unit = blockIdx.y * (kRowThreads / 32) + (threadIdx.x >> 5);   // K and V of every head
  if (unit >= 2 * c.batch * c.Hkv) return;
  const bool is_key = unit < c.batch * c.Hkv;
  const int bh = is_key ? unit : unit - c.batch * c.Hkv, b = bh / c.Hkv, h = bh - b * c.Hkv;
  constexpr int kAtOnce = 32 / kLanes, kTurns = kBlockRows / kAtOnce;   // rows that a warp has side by side
  const int chunk = lane % kLanes, sub = lane / kLanes;
  const int start = first ? first[c.per_head ? bh : b] : 0, n = paged_length(c, b, h);
  if (blockIdx.x == 0 && is_key && lane == 0) check_length(c, b, h);
  // blocks of the pages, so that a warp reads one of them: the first may begin before `start`
  const long long row0 = ((long long)start / kBlockRows - (start < 0 && start % kBlockRows != 0) + blockIdx.x) * kBlockRows;
  long long at = -1;
  if (row0 >= 0 && row0 < n) {
    at = paged_block(c, b, h, (int)(row0 / kBlockRows));
    if (at < 0 && lane == 0) atomicOr(c.dev_status, kDevBadIndex);
  }
  if (chunk * 8 >= c.d) return;
  const uint8_t* block = (is_key ? c.K : c.V) + (at < 0 ? 0 : at);
  T* out = (is_key ? K_out : V_out) + (long long)bh * n_rows * c.d + chunk * 8;
  const int m = chunk >> 2, q = chunk & 3, words = c.d >> 5;
  Pack8<T> raw[kTurns];
  uint32_t codes[kTurns], params[kTurns];
#pragma unroll
  for (int t = 0; t < kTurns; ++t) {
    const int r = t * kAtOnce + sub;
    raw[t].zero();
    codes[t] = params[t] = 0u;
    if (at < 0 || row0 + r >= n) continue;
    if constexpr (!kInt4) {
      raw[t].load(reinterpret_cast<const T*>(block + (long long)r * c.row_bytes) + chunk * 8);
    } else {
      const uint8_t* row = block + r * c.row_bytes;
      if (is_key) {
        codes[t] = reinterpret_cast<const unsigned int*>(row)[q * words + m];
      } else {
        const unsigned short* v = reinterpret_cast<const unsigned short*>(row);
        codes[t] = v[2 * q * words + m] | (unsigned int)v[(2 * q + 1) * words + m] << 16;
      }
      const unsigned short* p = reinterpret_cast<const unsigned short*>(block + int4_params(c.d, chunk * 8 / c.group, r));
      params[t] = p[0] | (unsigned int)p[4] << 16;
    }
  }
#pragma unroll
  for (int t = 0; t < kTurns; ++t) {
    const long long i = row0 + t * kAtOnce + sub - start;
    if (i < 0 || i >= n_rows) continue;
    if constexpr (!kInt4) {
      raw[t].put(out + i * c.d);
    } else {
      const float step = __uint_as_float(params[t] << 16), lo = __uint_as_float(params[t] & 0xFFFF0000u);
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        // 16 + code, by its bits; step * code is exact, so that there is one rounding
        const float code = __uint_as_float(((e < 5 ? codes[t] << (19 - 4 * e) : codes[t] >> (4 * e - 19)) & 0x00780000u) | 0x41800000u) - 16.f;
        x[e] = fmaf(step, code, lo);
      }
      Pack8<T>::store(out + i * c.d, x);
    }
  }
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
    return launch_chained(int4 ? paged_append_kernel<float, true, 2> : paged_append_kernel<float, false, 2>, grid, kRowThreads, 0, st, c, Kn,
                          Vn, K_pages, V_pages, positions, rot, Q, (float*)Q_out, lanes);
  return launch_chained(int4 ? paged_append_kernel<__nv_bfloat16, true, 3> : paged_append_kernel<__nv_bfloat16, false, 3>, grid, kRowThreads, 0,
                        st, c, Kn, Vn, K_pages, V_pages, positions, rot, Q, (__nv_bfloat16*)Q_out, lanes);
}

namespace {
template <typename T, bool kInt4> void (*pick_read(int lanes))(PagedCache, const int*, int, T*, T*) {
  switch (lanes) {
    case 4: return paged_read_kernel<T, kInt4, 4>;
    case 8: return paged_read_kernel<T, kInt4, 8>;
    case 16: return paged_read_kernel<T, kInt4, 16>;
    default: return paged_read_kernel<T, kInt4, 32>;
  }
}
template <typename T> cudaError_t launch_read_t(const PagedCache& c, const int* first, int n_rows, T* K_out, T* V_out, cudaStream_t st) {
  // 16 rows more than n_rows: the first block may begin before the first row
  const int units = 2 * c.batch * c.Hkv, warps = kRowThreads / 32;
  const dim3 grid((unsigned int)((n_rows + (first ? kBlockRows - 1 : 0) + kBlockRows - 1) / kBlockRows), (unsigned int)((units + warps - 1) / warps));
  const int lanes = lanes_per_row(c.d);
  return launch_chained(c.format == RESTKV_PAGES_INT4 ? pick_read<T, true>(lanes) : pick_read<T, false>(lanes), grid, kRowThreads, 0, st, c,
                        first, n_rows, K_out, V_out);
}
}  // namespace

cudaError_t launch_paged_read(const PagedCache& c, bool f32, const int* first, int n_rows, void* K_out, void* V_out, cudaStream_t st) {
  return f32 ? launch_read_t(c, first, n_rows, (float*)K_out, (float*)V_out, st)
             : launch_read_t(c, first, n_rows, (__nv_bfloat16*)K_out, (__nv_bfloat16*)V_out, st);
}

}  // namespace restkv
