// Rows into and out of the paged cache.
#include <type_traits>

#include "paged.cuh"
#include "sm100_ptx.cuh"

namespace restkv {

namespace {

constexpr int kRowThreads = 128;

// ---- 8 dims of a row (one thread's chunk) into 4 bits ----

// The group's offset and step; what cannot be quantised is set right first (a NaN, an infinity, 2^120 and more: rare, one vote).  By whole
// warps: a group lies in aligned threads.
__device__ __forceinline__ void int4_grid(float* x, int group, float* lo, float* step) {
  float probe = 0.f, l, h;
  auto range = [&]() {
    l = fminf(fminf(x[0], x[1]), fminf(x[2], x[3]));
    l = fminf(l, fminf(fminf(x[4], x[5]), fminf(x[6], x[7])));
    h = fmaxf(ptx::fmax3(ptx::fmax3(x[0], x[1], x[2]), x[3], x[4]), ptx::fmax3(x[5], x[6], x[7]));
  };
  range();
#pragma unroll
  for (int e = 0; e < 8; ++e) probe = fmaf(x[e], 0.f, probe);   // 0 unless one of them is not finite
  if (__any_sync(0xffffffffu, !(probe == 0.f) || h > 0x1p120f || l < -0x1p120f)) {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = int4_input(x[e]);
    range();
  }
  for (int off = 1; off < group / 8; off <<= 1) {
    l = fminf(l, __shfl_xor_sync(0xffffffffu, l, off));
    h = fmaxf(h, __shfl_xor_sync(0xffffffffu, h, off));
  }
  *lo = bf16_below(l);
  *step = bf16_above(__fdiv_rn(h - *lo, 15.f));
}

// The codes of 8 values, 4 bits each from the lowest on: the nearest one of (x - lo) / step, ties to even (common where the inputs are
// bf16).  A product with 1 / step finds it but for a neighbour near a tie; the remainder, which is exact, tells.  At most 15, since
// x - lo <= 15 step (1 + 2^-24).
__device__ __forceinline__ uint32_t int4_codes(const float* x, float lo, float step) {
  if (step < 0x1p-100f) {   // 1 / step could overflow; a group without span has step 0
    uint32_t w = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) w |= (step > 0.f ? (uint32_t)rintf(__fdiv_rn(x[e] - lo, step)) : 0u) << (4 * e);
    return w;
  }
  const float inv = __frcp_rn(step), half = 0.5f * step, below = __uint_as_float(__float_as_uint(half) - 1u);
  float sum[2] = {0.f, 0.f};   // c0 + 16 c1 + 256 c2 + 4096 c3 of both halves
#pragma unroll
  for (int e = 7; e >= 0; --e) {
    const float d = x[e] - lo;
    const float r = fmaf(d, inv, 12582912.f);          // 1.5 * 2^23: rounds to a whole number, ties to even
    float c = r - 12582912.f;
    const float rest = fmaf(-c, step, d);
    const float limit = __float_as_uint(r) & 1u ? below : half;   // an odd one gives way on a tie, too
    if (fabsf(rest) > limit) c += rest > 0.f ? 1.f : -1.f;
    sum[e >> 2] = fmaf(sum[e >> 2], 16.f, c);
  }
  return (uint32_t)sum[0] | (uint32_t)sum[1] << 16;
}

// grid (batch * n_tokens / warps, y): a warp takes a token, or with few tokens the y-th part of its rows, so that where the token goes and
// its cosines and sines are found once.  A row lies in kLanes threads, 32 / kLanes heads side by side; Q's heads, then K's, then V's,
// some rounds of them on their way before the first is needed.  What bounds it: in 16 bits HBM (658 MB of traffic for 8 x up to 4093 tokens,
// 6.0 TB/s; 100 MB of it are queries past a sequence's count, read and replaced by zeros); in 4 bits no unit alone (366 instructions per warp
// and 256 values, a quarter of them the codes: issue slots 68% and DRAM 47% busy with 40% of the warps); for one token the latency of
// lengths -> table -> row.  Measured, 32 + 8 heads of 128: one token 2.8 us; 8 x up to 4093 tokens, half of the dims rotated, into bf16
// 112 us; 32768 rotated tokens into 4 bits 176 us (730 MB at least: 4.1 TB/s), 2048 unrotated ones without queries 8.0 us.
struct AppendArgs {
  PagedCache c;
  RowsView K, V, Q;         // Q.data null: no queries
  uint8_t *K_pages, *V_pages;
  const int* positions;     // or null
  RotationView rot;
  void* Q_out;
};

// 72 registers, 28 warps per SM: with 80 (24 warps) or 64 (32 warps, some values found again) 2048 tokens into 4 bits and read back take as
// long and 10% longer, 8 x 4093 tokens into bf16 2% longer and 1%.
template <typename T, bool kInt4, int kLanes>
__global__ void __launch_bounds__(kRowThreads, 7) paged_append_kernel(const __grid_constant__ AppendArgs a) {
  ptx::grid_dependency_wait();
  ptx::grid_dependency_launch();
  constexpr int kAtOnce = 32 / kLanes;
  // rounds on their way together; quantising is long code, of which more copies cost instruction fetches
  constexpr int kAhead = sizeof(T) == 2 ? 4 : 2, kAheadKV = kInt4 ? 1 : kAhead;
  const PagedCache& c = a.c;
  const int lane = threadIdx.x & 31, chunk = lane % kLanes, sub = lane / kLanes;
  const long long token = (long long)blockIdx.x * (kRowThreads / 32) + (threadIdx.x >> 5);
  if (token >= (long long)c.batch * c.n_tokens) return;
  const int b = (int)(token / c.n_tokens), i = (int)token - b * c.n_tokens;
  const bool has = chunk * 8 < c.d;
  const int n_q = a.Q.data ? c.Hq : 0, q_rounds = (n_q + kAtOnce - 1) / kAtOnce, kv_rounds = (c.Hkv + kAtOnce - 1) / kAtOnce;
  const int rounds = q_rounds + 2 * kv_rounds;
  const int r0 = rounds * (int)blockIdx.y / (int)gridDim.y, r1 = rounds * ((int)blockIdx.y + 1) / (int)gridDim.y;

  const int count = paged_count(c, b);
  const bool there = i < count;
  const int per_page = c.page_rows / kBlockRows;
  int page = -1, block_of_page = 0, row_of_block = 0;
  auto find = [&](int h) {
    const long long row = (long long)c.lengths[c.per_head ? b * c.Hkv + h : b] - count + i;
    page = -1;
    if (row < 0 || row >= c.capacity()) return;
    const int slot_of_table = (int)row / c.page_rows, r = (int)row - slot_of_table * c.page_rows;
    page = c.table[(long long)b * c.table_width + slot_of_table];
    block_of_page = r / kBlockRows;
    row_of_block = r % kBlockRows;
  };
  if (there && !c.per_head) find(0);   // with lengths per head that is each head's own matter
  float cs[8], sn[8];
  const RotationView& rot = a.rot;
  bool turns = false, placed = true;
  if (there && rot.cos) {
    const int p = a.positions ? a.positions[token] : c.lengths[b] - count + i;
    placed = (unsigned int)p < (unsigned int)rot.n_positions;
    if (!placed && lane == 0) atomicOr(c.dev_status, kDevBadIndex);
    turns = placed && chunk * 8 < 2 * rot.half;
    if (turns) {
      // in halves 8 angles from the chunk's place in its half on, interleaved 4 of them twice
      const long long at = (long long)p * rot.half + (rot.interleaved ? chunk * 4 : chunk * 8 < rot.half ? chunk * 8 : chunk * 8 - rot.half);
      const float4 c0 = *reinterpret_cast<const float4*>(rot.cos + at), s0 = *reinterpret_cast<const float4*>(rot.sin + at);
      if (rot.interleaved) {
        cs[0] = cs[1] = c0.x; cs[2] = cs[3] = c0.y; cs[4] = cs[5] = c0.z; cs[6] = cs[7] = c0.w;
        sn[0] = sn[1] = s0.x; sn[2] = sn[3] = s0.y; sn[4] = sn[5] = s0.z; sn[6] = sn[7] = s0.w;
      } else {
        const float4 c1 = *reinterpret_cast<const float4*>(rot.cos + at + 4), s1 = *reinterpret_cast<const float4*>(rot.sin + at + 4);
        cs[0] = c0.x; cs[1] = c0.y; cs[2] = c0.z; cs[3] = c0.w; cs[4] = c1.x; cs[5] = c1.y; cs[6] = c1.z; cs[7] = c1.w;
        sn[0] = s0.x; sn[1] = s0.y; sn[2] = s0.z; sn[3] = s0.w; sn[4] = s1.x; sn[5] = s1.y; sn[6] = s1.z; sn[7] = s1.w;
        if (chunk * 8 < rot.half) {   // the first of a pair: a cos - b sin; the second: b cos + a sin
#pragma unroll
          for (int e = 0; e < 8; ++e) sn[e] = -sn[e];
        }
      }
    }
  }
  const int half_chunks = rot.half >> 3;
  const int partner = (lane + (rot.interleaved || !turns ? 0 : chunk < half_chunks ? half_chunks : -half_chunks)) & 31;
  // products and sums are rounded one by one, as they are stated
  auto rotate = [&](const Pack8<T>& own, float* x) {   // by whole warps: they exchange halves
    if (!rot.cos) return;
    if (rot.interleaved) {
      if (!turns) return;
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        const float u = x[e], v = x[e + 1];
        x[e] = __fsub_rn(__fmul_rn(u, cs[e]), __fmul_rn(v, sn[e]));
        x[e + 1] = __fadd_rn(__fmul_rn(v, cs[e]), __fmul_rn(u, sn[e]));
      }
    } else {
      float other[8];
      own.exchange(partner, other);
      if (!turns) return;
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = __fadd_rn(__fmul_rn(x[e], cs[e]), __fmul_rn(other[e], sn[e]));
    }
  };
  // Rounds [from, to) of `heads` heads whose rows lie `stride` elements apart; (rows past a count are loaded, too: they are the caller's)
  auto pass = [&](auto ahead, int from, int to, const RowsView& rows, int heads, auto&& take) {
    constexpr int kUnroll = decltype(ahead)::value;
    if (from >= to) return;
    const T* src = reinterpret_cast<const T*>(rows.data) + b * rows.sb + i * rows.sn + chunk * 8 + (from * kAtOnce + sub) * rows.sh;
    const long long step = kAtOnce * rows.sh;
    int left = has ? heads - sub - from * kAtOnce : 0;   // heads from this thread's on
    for (int r = from; r < to; r += kUnroll) {
      Pack8<T> raw[kUnroll];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        raw[u].zero();
        if (r + u < to && left > u * kAtOnce) raw[u].load(src + u * step);
      }
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        if (r + u >= to) break;
        take(raw[u], (r + u) * kAtOnce + sub, left > u * kAtOnce);
      }
      src += kUnroll * step;
      left -= kUnroll * kAtOnce;
    }
  };
  {
    T* const to = reinterpret_cast<T*>(a.Q_out) + ((long long)b * c.Hq * c.n_tokens + i) * c.d + chunk * 8;
    const long long row = (long long)c.n_tokens * c.d;
    pass(std::integral_constant<int, kAhead>{}, r0, r1 < q_rounds ? r1 : q_rounds, a.Q, n_q, [&](Pack8<T>& raw, int h, bool mine) {
      float x[8];
      raw.get(x);
      rotate(raw, x);
      if (!mine || !placed) return;
      if (there) {
        Pack8<T>::store(to + h * row, x);
      } else {
        Pack8<T> none;
        none.zero();
        none.put(to + h * row);
      }
    });
  }
  if (!there || !placed) return;
  if (!c.per_head && (unsigned int)page >= (unsigned int)c.n_pages) {
    if (lane == 0 && r1 > q_rounds) atomicOr(c.dev_status, kDevBadIndex);
    return;
  }
  // where the chunk goes: the block in head 0's pages, and in it the key's and the value's codes, step and offset
  long long block = 0;
  int at_key = 0, at_value = 0, at_params = 0;
  const int m = chunk >> 2, q = chunk & 3, words = c.d >> 5;
  const bool leads = kInt4 && (chunk * 8 & (c.group - 1)) == 0;
  auto place = [&]() {
    block = (long long)page * c.Hkv * c.head_bytes + (long long)block_of_page * c.block_bytes;
    const int row = row_of_block * c.row_bytes;
    at_key = row + (kInt4 ? (q * words + m) * 4 : chunk * 8 * (int)sizeof(T));
    at_value = kInt4 ? row + (2 * q * words + m) * 2 : at_key;
    if (kInt4) at_params = int4_params(c.d, chunk * 8 / c.group, row_of_block);
  };
  if (!c.per_head) place();
  auto store = [&](auto key, Pack8<T>& raw, int h, bool mine) {
    constexpr bool kKey = decltype(key)::value;
    float x[8];
    raw.get(x);
    if (kKey) rotate(raw, x);
    float lo, step;
    if constexpr (kInt4) int4_grid(x, c.group, &lo, &step);
    if (!mine) return;
    if (c.per_head) {
      find(h);
      if ((unsigned int)page >= (unsigned int)c.n_pages) {
        if (chunk == 0) atomicOr(c.dev_status, kDevBadIndex);
        return;
      }
      place();
    }
    uint8_t* const to = (kKey ? a.K_pages : a.V_pages) + block + h * c.head_bytes;
    if constexpr (kInt4) {
      const uint32_t w = int4_codes(x, lo, step);
      if (kKey) {
        *reinterpret_cast<unsigned int*>(to + at_key) = w;
      } else {
        unsigned short* const v = reinterpret_cast<unsigned short*>(to + at_value);
        v[0] = (unsigned short)(w & 0xFFFFu);
        v[words] = (unsigned short)(w >> 16);
      }
      if (leads) {
        unsigned short* const p = reinterpret_cast<unsigned short*>(to + at_params);
        p[0] = (unsigned short)(__float_as_uint(step) >> 16);
        p[4] = (unsigned short)(__float_as_uint(lo) >> 16);
      }
    } else {
      Pack8<T>::store(reinterpret_cast<T*>(to + at_key), x);
    }
  };
  const int k0 = r0 - q_rounds, k1 = r1 - q_rounds, v0 = k0 - kv_rounds, v1 = k1 - kv_rounds;
  const std::integral_constant<int, kAheadKV> few;
  pass(few, k0 > 0 ? k0 : 0, k1 < kv_rounds ? k1 : kv_rounds, a.K, c.Hkv, [&](Pack8<T>& raw, int h, bool mine) { store(std::true_type{}, raw, h, mine); });
  pass(few, v0 > 0 ? v0 : 0, v1 < kv_rounds ? v1 : kv_rounds, a.V, c.Hkv, [&](Pack8<T>& raw, int h, bool mine) { store(std::false_type{}, raw, h, mine); });
}

// ---- reading back ----

// 8 values of a group from their codes: offset + step * code, rounded once.
__device__ __forceinline__ void int4_read(uint32_t w, uint32_t step_hi, uint32_t lo_hi, float* out) {   // step, offset as fp32 bits
  float x[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    // 16 + code, by its bits
    const float code = __uint_as_float(((e < 5 ? w << (19 - 4 * e) : w >> (4 * e - 19)) & 0x00780000u) | 0x41800000u) - 16.f;
    x[e] = fmaf(__uint_as_float(step_hi), code, __uint_as_float(lo_hi));
  }
  Pack8<float>::store(out, x);
}
__device__ __forceinline__ void int4_read(uint32_t w, uint32_t step_hi, uint32_t lo_hi, __nv_bfloat16* out) {
  // in pairs: 128 + code, 128 off again, then one fused operation, which rounds step * code + offset as a whole
  const uint32_t ss = __byte_perm(step_hi, 0u, 0x3232), ll = __byte_perm(lo_hi, 0u, 0x3232);
  uint32_t p[4];   // dims i, i + 4
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t c = (w >> (4 * i) & 0x000F000Fu) | 0x43004300u;
    asm("add.rn.bf16x2 %0, %0, %1;" : "+r"(c) : "r"(0xC300C300u));
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(p[i]) : "r"(ss), "r"(c), "r"(ll));
  }
  *reinterpret_cast<uint4*>(out) = make_uint4(__byte_perm(p[0], p[1], 0x5410), __byte_perm(p[2], p[3], 0x5410), __byte_perm(p[0], p[1], 0x7632),
                                              __byte_perm(p[2], p[3], 0x7632));
}

// grid (runs of `run` blocks of 16 rows, batch * Hkv / warps): a warp takes such a run of a head, K and V, so that a block's page is
// looked up once and its loads are on their way together.  Rows first .. first + n_rows of every head; first may be negative.  Bound by HBM (the rows written).
// Measured, 4-bit rows into bf16: 8 x up to 32749 rows 221 us (5.8 TB/s), 2176 rows 4.1 us.
// (4 blocks a run: the set-up is a fifth of the instructions.  With few rows 1, until there are 8 warps per SM: 2176 rows 5.0 us, 8.7 in runs
// of 4.)
template <typename T, bool kInt4, int kLanes>
__global__ void __launch_bounds__(kRowThreads) paged_read_kernel(const PagedCache c, const int* __restrict__ first, int n_rows, T* K_out,
                                                                 T* V_out, int run) {
  ptx::grid_dependency_wait();
  ptx::grid_dependency_launch();
  const int lane = threadIdx.x & 31, bh = blockIdx.y * (kRowThreads / 32) + (threadIdx.x >> 5);
  if (bh >= c.batch * c.Hkv) return;
  const int b = bh / c.Hkv, h = bh - b * c.Hkv;
  constexpr int kAtOnce = 32 / kLanes, kTurns = kBlockRows / kAtOnce;   // rows that a warp has side by side
  const int chunk = lane % kLanes, sub = lane / kLanes;
  const int start = first ? first[c.per_head ? bh : b] : 0, n = paged_length(c, b, h);
  if (blockIdx.x == 0 && lane == 0) check_length(c, b, h);
  // blocks of the pages, so that a warp reads whole ones: the first may begin before `start`.  `shift`: out's row of the run's first
  const long long row0 = ((long long)(start >> 4) + (long long)blockIdx.x * run) * kBlockRows;
  const long long shift = row0 - start;
  if (shift >= n_rows) return;
  const int per_page = c.page_rows / kBlockRows;
  int slot = 0, within = 0;
  if (row0 >= 0 && row0 < n) {
    slot = (int)(row0 / kBlockRows) / per_page;
    within = (int)(row0 / kBlockRows) - slot * per_page;
  }
  const int m = chunk >> 2, q = chunk & 3, words = c.d >> 5;
  const bool has = chunk * 8 < c.d;
  T* const k_to = K_out + ((long long)bh * n_rows + shift) * c.d + chunk * 8;
  T* const v_to = V_out + ((long long)bh * n_rows + shift) * c.d + chunk * 8;
#pragma unroll 1
  for (int k = 0; k < run; ++k) {
    // rows of the block that are there, and rows of the output that it covers
    const long long block_row = row0 + k * kBlockRows;
    const int left = block_row < 0 ? 0 : block_row >= n ? 0 : n - block_row < kBlockRows ? (int)(n - block_row) : kBlockRows;
    const int from = shift + k * kBlockRows < 0 ? (int)-(shift + k * kBlockRows) : 0;
    const long long room = n_rows - (shift + k * kBlockRows);
    if (room <= 0) return;
    const int to = room < kBlockRows ? (int)room : kBlockRows;
    long long at = -1;
    if (left > 0) {
      const int page = c.table[(long long)b * c.table_width + slot];
      if ((unsigned int)page < (unsigned int)c.n_pages) at = (((long long)page * c.Hkv + h) * per_page + within) * c.block_bytes;
      else if (lane == 0) atomicOr(c.dev_status, kDevBadIndex);
    }
    if (block_row >= 0 && ++within == per_page) { within = 0; ++slot; }   // (a run may begin before row 0, at block 0 of slot 0)
    if (!has) continue;
#pragma unroll
    for (int side = 0; side < 2; ++side) {
      T* const out = (side == 0 ? k_to : v_to) + k * kBlockRows * c.d;
      if (at < 0) {
        Pack8<T> none;
        none.zero();
        for (int r = sub; r < to; r += kAtOnce)
          if (r >= from) none.put(out + r * c.d);
        continue;
      }
      const uint8_t* block = (side == 0 ? c.K : c.V) + at;
      if constexpr (!kInt4) {
        Pack8<T> raw[kTurns];
#pragma unroll
        for (int t = 0; t < kTurns; ++t) {
          const int r = t * kAtOnce + sub;
          raw[t].zero();
          if (r < left) raw[t].load(reinterpret_cast<const T*>(block + r * c.row_bytes) + chunk * 8);
        }
#pragma unroll
        for (int t = 0; t < kTurns; ++t) {
          const int r = t * kAtOnce + sub;
          if (r >= from && r < to) raw[t].put(out + r * c.d);
        }
      } else {
        // steps and offsets of rows r % 4 + 4 j come in one load
        constexpr int kLoads = kAtOnce >= 4 ? 1 : 4 / kAtOnce;
        const uint8_t* params = block + 8 * c.d + 64 * (chunk * 8 / c.group);
        uint4 u[kLoads];
        uint32_t w[kTurns];
#pragma unroll
        for (int x = 0; x < kLoads; ++x) u[x] = *reinterpret_cast<const uint4*>(params + 16 * ((x * kAtOnce + sub) & 3));
#pragma unroll
        for (int t = 0; t < kTurns; ++t) {
          const uint8_t* row = block + (t * kAtOnce + sub) * c.row_bytes;
          if (side == 0) {
            w[t] = reinterpret_cast<const unsigned int*>(row)[q * words + m];
          } else {
            const unsigned short* v = reinterpret_cast<const unsigned short*>(row);
            w[t] = v[2 * q * words + m] | (unsigned int)v[(2 * q + 1) * words + m] << 16;
          }
        }
#pragma unroll
        for (int t = 0; t < kTurns; ++t) {
          const int r = t * kAtOnce + sub;
          if (r < from || r >= to) continue;
          const uint4 p = u[t % kLoads];
          const int j = kAtOnce == 8 ? 2 * t + (sub >> 2) : t * kAtOnce / 4;
          const uint32_t s = j & 2 ? p.y : p.x, l = j & 2 ? p.w : p.z;
          const bool there = r < left;
          int4_read(there ? w[t] : 0u, there ? (j & 1 ? s & 0xFFFF0000u : s << 16) : 0u, there ? (j & 1 ? l & 0xFFFF0000u : l << 16) : 0u,
                    out + r * c.d);
        }
      }
    }
  }
}

template <typename T, bool kInt4> void (*pick_append(int lanes))(AppendArgs) {
  switch (lanes) {
    case 4: return paged_append_kernel<T, kInt4, 4>;
    case 8: return paged_append_kernel<T, kInt4, 8>;
    case 16: return paged_append_kernel<T, kInt4, 16>;
    default: return paged_append_kernel<T, kInt4, 32>;
  }
}

}  // namespace

cudaError_t launch_paged_append(const PagedCache& c, bool f32, const RowsView& Kn, const RowsView& Vn, uint8_t* K_pages, uint8_t* V_pages,
                                const int* positions, const RotationView& rot, const RowsView& Q, void* Q_out, int sm_count, cudaStream_t st) {
  const int lanes = lanes_per_row(c.d), at_once = 32 / lanes, warps = kRowThreads / 32;
  const AppendArgs a{c, Kn, Vn, Q, K_pages, V_pages, positions, rot, Q_out};
  const long long blocks = ((long long)c.batch * c.n_tokens + warps - 1) / warps;
  // a warp per token finds its place and its angles once; with few tokens the rows go to warps of their own until there are 16 per SM
  // (2048 tokens into 4 bits and read back 14.0 us; until there are 32, 64: 14.5, 15.3)
  const int rounds = ((Q.data ? c.Hq : 0) + at_once - 1) / at_once + 2 * ((c.Hkv + at_once - 1) / at_once);
  long long y = (4LL * sm_count + blocks - 1) / blocks;
  if (y > rounds) y = rounds;
  const bool int4 = c.format == RESTKV_PAGES_INT4;
  void (*kernel)(AppendArgs) = f32 ? (int4 ? pick_append<float, true>(lanes) : pick_append<float, false>(lanes))
                                   : (int4 ? pick_append<__nv_bfloat16, true>(lanes) : pick_append<__nv_bfloat16, false>(lanes));
  return launch_chained(kernel, dim3((unsigned int)blocks, (unsigned int)y), kRowThreads, 0, st, a);
}

namespace {
template <typename T, bool kInt4> void (*pick_read(int lanes))(PagedCache, const int*, int, T*, T*, int) {
  switch (lanes) {
    case 4: return paged_read_kernel<T, kInt4, 4>;
    case 8: return paged_read_kernel<T, kInt4, 8>;
    case 16: return paged_read_kernel<T, kInt4, 16>;
    default: return paged_read_kernel<T, kInt4, 32>;
  }
}
template <typename T> cudaError_t launch_read_t(const PagedCache& c, const int* first, int n_rows, T* K_out, T* V_out, int sm_count, cudaStream_t st) {
  // 15 rows more than n_rows: the first block may begin before the first row
  const int warps = kRowThreads / 32;
  const long long blocks = ((long long)n_rows + (first ? kBlockRows - 1 : 0) + kBlockRows - 1) / kBlockRows;
  const int run = blocks * c.batch * c.Hkv >= 4 * 8LL * sm_count ? 4 : 1;
  const dim3 grid((unsigned int)((blocks + run - 1) / run),
                  (unsigned int)((c.batch * c.Hkv + warps - 1) / warps));
  const int lanes = lanes_per_row(c.d);
  return launch_chained(c.format == RESTKV_PAGES_INT4 ? pick_read<T, true>(lanes) : pick_read<T, false>(lanes), grid, kRowThreads, 0, st, c,
                        first, n_rows, K_out, V_out, run);
}
}  // namespace

cudaError_t launch_paged_read(const PagedCache& c, bool f32, const int* first, int n_rows, void* K_out, void* V_out, int sm_count,
                              cudaStream_t st) {
  return f32 ? launch_read_t(c, first, n_rows, (float*)K_out, (float*)V_out, sm_count, st)
             : launch_read_t(c, first, n_rows, (__nv_bfloat16*)K_out, (__nv_bfloat16*)V_out, sm_count, st);
}

}  // namespace restkv
