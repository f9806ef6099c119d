// The paged cache: its description as the kernels get it, where a row lies, and the 4-bit format.
#pragma once

#include "restkv_common.cuh"

namespace restkv {

constexpr int kBlockRows = 16;   // rows of a block: what one tile of the attention kernels holds, and a 4-bit block's parameters

struct PagedCache {
  int batch, Hq, Hkv, G, d;
  int format, group;
  int page_rows, n_pages, table_width;
  int per_head;               // lengths [batch, Hkv] instead of [batch]
  float scale, softcap;       // softcap 0: none
  int row_bytes;              // of a row of elements, or of a row's codes
  int block_bytes;            // 16 rows (and their steps and offsets)
  long long head_bytes;       // one head's rows of a page
  const int* lengths;
  const int* table;
  const int* counts;          // null: every sequence has n_tokens
  int n_tokens;
  const uint8_t *K, *V;
  unsigned int* dev_status;

  __host__ __device__ long long capacity() const { return (long long)table_width * page_rows; }
};

// Threads that a row takes, 8 dims each: a power of two.
inline int lanes_per_row(int d) {
  int lanes = 4;
  while (lanes * 8 < d) lanes *= 2;
  return lanes;
}

struct RowsView {   // [batch, heads, n_tokens, d] in element strides
  const void* data;
  long long sb, sh, sn;
};

struct RotationView {
  const float *cos, *sin;   // null: no rotation
  int n_positions, half;    // rotary_dim / 2
  int interleaved;
};

// Rows of a sequence for one KV head: within the table, and never negative.
__device__ __forceinline__ int paged_length(const PagedCache& c, int b, int h) {
  const int n = c.lengths[c.per_head ? b * c.Hkv + h : b];
  const long long most = c.capacity();
  return n < 0 ? 0 : (int)(n < most ? n : most);
}
// Sets the sticky status if a sequence claims more rows than its table can name.
__device__ __forceinline__ void check_length(const PagedCache& c, int b, int h) {
  if (c.lengths[c.per_head ? b * c.Hkv + h : b] > c.capacity()) atomicOr(c.dev_status, kDevBadIndex);
}
__device__ __forceinline__ int paged_count(const PagedCache& c, int b) {
  if (!c.counts) return c.n_tokens;
  const int n = c.counts[b];
  return n < 0 ? 0 : n < c.n_tokens ? n : c.n_tokens;
}
// Block `block` of 16 rows of a sequence and head, counted from the first of the pool, in K's pages as in V's; -1 if the table's entry is
// out of range.
__device__ __forceinline__ int paged_block_index(const PagedCache& c, int b, int h, int block) {
  const int per_page = c.page_rows / kBlockRows;
  const int slot = block / per_page;
  const int page = c.table[(long long)b * c.table_width + slot];
  if ((unsigned int)page >= (unsigned int)c.n_pages) return -1;
  return (page * c.Hkv + h) * per_page + block - slot * per_page;
}
// The same as a byte offset.
__device__ __forceinline__ long long paged_block(const PagedCache& c, int b, int h, int block) {
  const int at = paged_block_index(c, b, h, block);
  return at < 0 ? -1 : (long long)at * c.block_bytes;
}

// ---- the 4-bit format ----
// Offset and step of a group are bf16, rounded outward so that offset <= every value <= offset + 15 * step: the codes clip nothing
// and the error of a value is half a step, also where a group lies far from 0.  (A symmetric grid would spend half its codes on nothing there.)
__device__ __forceinline__ float bf16_below(float x) {
  const unsigned int u = __float_as_uint(x), t = u & 0xFFFF0000u;
  return __uint_as_float(u != t && (int)u < 0 ? t + 0x10000u : t);
}
__device__ __forceinline__ float bf16_above(float x) {   // x >= 0
  const unsigned int u = __float_as_uint(x), t = u & 0xFFFF0000u;
  return __uint_as_float(u != t ? t + 0x10000u : t);
}
__device__ __forceinline__ float int4_input(float x) {   // NaN -> 0; 2^120 keeps the span of a group finite
  return x == x ? fminf(fmaxf(x, -0x1p120f), 0x1p120f) : 0.f;
}
// Byte of a block where row r has the step of group g; its offset lies 8 bytes on.
__device__ __forceinline__ int int4_params(int d, int g, int r) { return 8 * d + 64 * g + 16 * (r & 3) + 2 * (r >> 2); }

template <typename T> struct Pack8;   // 8 consecutive elements of a row
template <> struct Pack8<__nv_bfloat16> {
  uint4 u;
  __device__ void load(const __nv_bfloat16* p) { u = *reinterpret_cast<const uint4*>(p); }
  __device__ void zero() { u = make_uint4(0u, 0u, 0u, 0u); }
  __device__ void put(__nv_bfloat16* p) const { *reinterpret_cast<uint4*>(p) = u; }
  __device__ void exchange(int lane, float* x) const {   // another lane's, by the whole warp
    Pack8 o;
    o.u = make_uint4(__shfl_sync(0xffffffffu, u.x, lane), __shfl_sync(0xffffffffu, u.y, lane), __shfl_sync(0xffffffffu, u.z, lane),
                     __shfl_sync(0xffffffffu, u.w, lane));
    o.get(x);
  }
  __device__ void get(float* x) const {
    const unsigned int w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(w[i] << 16);
      x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
  }
  __device__ static void store(__nv_bfloat16* p, const float* x) {
    uint4 v;
    unsigned int* w = &v.x;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 pair = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
      w[i] = *reinterpret_cast<const unsigned int*>(&pair);
    }
    *reinterpret_cast<uint4*>(p) = v;
  }
};
template <> struct Pack8<float> {
  float4 a, b;
  __device__ void load(const float* p) { a = reinterpret_cast<const float4*>(p)[0]; b = reinterpret_cast<const float4*>(p)[1]; }
  __device__ void zero() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
  __device__ void put(float* p) const { reinterpret_cast<float4*>(p)[0] = a; reinterpret_cast<float4*>(p)[1] = b; }
  __device__ void exchange(int lane, float* x) const {
    float y[8];
    get(y);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = __shfl_sync(0xffffffffu, y[e], lane);
  }
  __device__ void get(float* x) const {
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
  }
  __device__ static void store(float* p, const float* x) {
    reinterpret_cast<float4*>(p)[0] = make_float4(x[0], x[1], x[2], x[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(x[4], x[5], x[6], x[7]);
  }
};

// 8 dims of a row of K or V, as fp32.
template <typename T, bool kInt4>
__device__ __forceinline__ void load_chunk(const PagedCache& c, const uint8_t* block, int r, int chunk, bool is_key, float* x) {
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
    for (int e = 0; e < 8; ++e) x[e] = fmaf(step, (float)(w >> (4 * e) & 15u), lo);
  }
}

// ---- launches ----
cudaError_t launch_paged_append(const PagedCache& c, bool f32, const RowsView& K_new, const RowsView& V_new, uint8_t* K_pages,
                                uint8_t* V_pages, const int* positions, const RotationView& rotation, const RowsView& Q, void* Q_out,
                                int sm_count, cudaStream_t st);
cudaError_t launch_paged_read(const PagedCache& c, bool f32, const int* first, int n_rows, void* K_out, void* V_out, int sm_count,
                              cudaStream_t st);
// fp32 SIMT attention: every dtype, format and head_dim.
int paged_simt_splits(const PagedCache& c, int sm_count);
size_t paged_simt_bytes(const PagedCache& c, int sm_count);
cudaError_t launch_paged_simt(const PagedCache& c, bool f32, const RowsView& Q, void* out, float* lse, float* part, int splits,
                              cudaStream_t st);
// bf16 with head_dim 64, 128 or 256 on the tensor pipe, up to 16 query rows per pass over the cache.
cudaError_t paged_mma_init(int (*clusters_of)[5]);
bool paged_mma_shape(const PagedCache& c);       // by type and head_dim alone
bool paged_mma_supported(const PagedCache& c);
size_t paged_mma_bytes(const PagedCache& c, int sm_count);
cudaError_t launch_paged_mma(void* state, const PagedCache& c, const RowsView& Q, void* out, float* lse, float* part, int sm_count,
                             const int (*clusters_of)[5], long long wait_limit, cudaStream_t st, int* launches);
// bf16 with head_dim 64 or 128 on tcgen05, 256 query rows of a KV head per pass: for at least kChunkRows of them, and kChunkAll in the call.
// A pass costs the same for few rows, and a call some 25 us before and after its passes.  Measured, 32 heads of 128 (8 KV heads), 4-bit rows,
// this one and the kernel for few tokens: 1 x 2200 rows, 48 tokens 30.1 and 29.5 us, 128 tokens 37.4 and 55.1; 1 x 17000 rows, 32 tokens 61
// and 55, 48 tokens 53 and 81; 8 x 4000 rows, 8 tokens 77 and 45, 16 tokens 78 and 75, 24 tokens 76 and 104.
constexpr int kChunkRows = 64, kChunkAll = 1536;
cudaError_t paged_chunk_init();
bool paged_chunk_shape(const PagedCache& c);     // by type, head_dim and query rows
bool paged_chunk_supported(const PagedCache& c);
size_t paged_chunk_bytes(const PagedCache& c, int sm_count);
cudaError_t launch_paged_chunk(const PagedCache& c, const RowsView& Q, void* out, float* lse, float* part, int sm_count, long long wait_limit,
                               cudaStream_t st);

}  // namespace restkv
