// What the tensor-core kernels of the cross attention share: K and V as they lie, for TMA; the merge of what several CTAs left of a unit.
#pragma once

#include <math.h>

#include "cross.cuh"
#include "paged_deal.cuh"

namespace restkv {
namespace {


// Whether rows can be described by a tensor map: strides that are no smaller than a row, nor past its 40 bits of bytes.
inline bool cross_map_fits(const CrossProblem& c, const RowsView& v) {
  for (long long st : {v.sb, v.sh, v.sn})
    if (st < c.d || st >= 1ll << 38) return false;
  return true;
}

// Boxes of box_rows rows and 64 dims of [sources, Hkv, n_rows, d]; rows past n_rows are filled with zeros.
inline bool make_cross_map(TcState* st, CUtensorMap* map, const CrossProblem& c, const RowsView& v, cuuint32_t box_rows) {
  const cuuint64_t dims[4] = {(cuuint64_t)c.d, (cuuint64_t)c.n_rows, (cuuint64_t)c.Hkv, (cuuint64_t)c.sources};
  const cuuint64_t str[3] = {(cuuint64_t)v.sn * 2, (cuuint64_t)v.sh * 2, (cuuint64_t)v.sb * 2};
  return encode_tiles(st, map, v.data, 4, dims, str, box_rows) == CUDA_SUCCESS;
}

// Tiles of all units (source, KV head, kRows query rows) end to end are dealt out over CTAs; each says in `begins` which unit and tile of it its run
// begins with (-1: none), and leaves what it has of a unit that it shares in one of two slots: o, fp32, and (m, l) of each row; the first
// for the unit that its run goes on with, the second for one that it begins.  What there is of a unit is merged by the blocks of the first CTA that
// began inside it (x; the one before it began the unit).
struct Shared {
  int unit, x, pieces;         // pieces 0: nothing for this block to do
  int b, h, rho0;
};
// Blocks (x of the grid) are CTAs of the kernel before, or units.  By blocks of 256 threads.
template <bool kByUnit>
__device__ __forceinline__ Shared shared_unit(const CrossProblem& c, const int2* begins, int ctas, int row_tiles, int rows) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  Shared s{(int)blockIdx.x, (int)blockIdx.x, 0, 0, 0, 0};
  auto inside = [&](int x) {
    const int2 o = x < ctas ? __ldcg(begins + x) : make_int2(-1, 0);
    return o.x == s.unit && o.y > 0;
  };
  if constexpr (kByUnit) {     // which CTAs began inside the unit: a bit each, two words per warp
    static_assert(kMaxCtas <= 512, "two CTAs per thread");
    __shared__ int inside_s[16];
    const unsigned int in0 = __ballot_sync(0xffffffffu, inside(warp * 64 + lane)), in1 = __ballot_sync(0xffffffffu, inside(warp * 64 + 32 + lane));
    if (lane < 2) inside_s[2 * warp + lane] = (int)(lane ? in1 : in0);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const unsigned int in = (unsigned int)inside_s[i];
      if (in && s.pieces == 0) s.x = 32 * i + __ffs((int)in) - 1;
      s.pieces += __popc(in);
    }
    if (s.pieces == 0) return s;
  } else {
    const int2 mine = __ldcg(begins + s.x), before = s.x > 0 ? __ldcg(begins + s.x - 1) : make_int2(-1, 0);
    s.unit = mine.x;
    if (mine.x < 0 || mine.y == 0 || (before.x == mine.x && before.y > 0)) return s;
    for (int n = 32; n == 32; s.pieces += n) n = __popc(__ballot_sync(0xffffffffu, inside(s.x + s.pieces + lane)));
  }
  ++s.pieces;                  // what the CTA before has of it
  const int bh = s.unit / row_tiles;
  s.b = bh / c.Hkv;
  s.h = bh - s.b * c.Hkv;
  s.rho0 = (s.unit - bh * row_tiles) * rows;
  return s;
}
// Piece k of the unit, in slots of `slot` floats.
__device__ __forceinline__ const float* piece_of(const Shared& u, const float* part, int k, long long slot) { return part + (2ll * (u.x - 1 + k) + (k == 0)) * slot; }

// Where a slot of kRows rows has float4 z of a row: rows of kD floats for few rows, [kD / 4, rows, 4] (as tensor memory is read) for many.
template <int kD, int kRows>
__device__ __forceinline__ int slot_at(int row, int z) {
  return kRows <= 32 ? row * kD + z : (z / 4 * kRows + row) * 4 + z % 4;
}

// grid (units or CTAs of the kernel before, row groups), block 256: kAtOnce rows by a warp, or, of few units with many pieces, by the eight warps of a
// block, each with every eighth piece, which merge in shared memory.  Two pieces of two rows asked for together (2048 query rows over 8192 rows, all of the
// call: 251 us; four pieces of two rows 259, four of four 270: fewer blocks at once; one piece of four 252).  One query group of 40 rows over 30000 rows, by
// pieces: 43.5 us, without the split 105.
template <int kD, int kRows, int kAtOnce, int kAhead, bool kByUnit>
__global__ void __launch_bounds__(256) cross_merge_kernel(const CrossProblem c, const float* __restrict__ part, const int2* __restrict__ begins, int ctas, int row_tiles) {
  grid_dependency_wait();
  grid_dependency_launch();
  constexpr int kPer = kD / 32, kWays = kByUnit ? 8 : 1;
  constexpr long long kSlot = kRows * (kD + 2);
  const Shared u = shared_unit<kByUnit>(c, begins, ctas, row_tiles, kRows);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int row0 = (kByUnit ? (int)blockIdx.y : 8 * (int)blockIdx.y + warp) * kAtOnce, left = (int)c.rows() - u.rho0 - row0;
  if (u.pieces == 0 || left <= 0) return;
  float mm[kAtOnce], ll[kAtOnce], acc[kAtOnce][kPer];
#pragma unroll
  for (int i = 0; i < kAtOnce; ++i) {
    mm[i] = -INFINITY;
    ll[i] = 0.f;
#pragma unroll
    for (int z = 0; z < kPer; ++z) acc[i][z] = 0.f;
  }
  auto load = [&](int k, int i, float2& ml, float (&o)[kPer]) {
    const float* const slot = piece_of(u, part, k, kSlot);
    const float* const from = slot + slot_at<kD, kRows>(row0 + i, kPer * lane);
    ml = __ldcg(reinterpret_cast<const float2*>(slot + kRows * kD) + row0 + i);
    if constexpr (kPer == 4) {
      const float4 v = __ldcg(reinterpret_cast<const float4*>(from));
      o[0] = v.x; o[1] = v.y; o[2] = v.z; o[3] = v.w;
    } else {
      const float2 v = __ldcg(reinterpret_cast<const float2*>(from));
      o[0] = v.x; o[1] = v.y;
    }
  };
  auto join = [&](int i, float2 ml, const float (&o)[kPer]) {
    // (no branch: a sum that is no number stays none, whatever its reference)
    const float top = fmaxf(mm[i], ml.x), down = mm[i] == -INFINITY ? 0.f : ex2_approx(mm[i] - top), f = ml.x == -INFINITY ? 0.f : ex2_approx(ml.x - top);
    mm[i] = top;
    ll[i] = fmaf(ll[i], down, ml.y * f);
#pragma unroll
    for (int z = 0; z < kPer; ++z) acc[i][z] = fmaf(acc[i][z], down, o[z] * f);
  };
  for (int k0 = kByUnit ? warp : 0; k0 < u.pieces; k0 += kWays * kAhead) {
    float2 ml[kAhead][kAtOnce];
    float o[kAhead][kAtOnce][kPer];
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i)
        if (k0 + kWays * j < u.pieces && i < left) load(k0 + kWays * j, i, ml[j][i], o[j][i]);
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i)
        if (k0 + kWays * j < u.pieces && i < left) join(i, ml[j][i], o[j][i]);
  }
  if constexpr (kByUnit) {
    __shared__ float2 ml_s[8][kAtOnce];
    __shared__ float acc_s[8][kAtOnce][kD];
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      if (lane == 0) ml_s[warp][i] = make_float2(mm[i], ll[i]);
#pragma unroll
      for (int z = 0; z < kPer; ++z) acc_s[warp][i][kPer * lane + z] = acc[i][z];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {                  // row i by warp i
      if (i != warp) continue;
      for (int w = 0; w < 8; ++w) {
        if (w == warp) continue;
        float o[kPer];
#pragma unroll
        for (int z = 0; z < kPer; ++z) o[z] = acc_s[w][i][kPer * lane + z];
        join(i, ml_s[w][i], o);
      }
    }
  }
#pragma unroll
  for (int i = 0; i < kAtOnce; ++i) {
    if (i >= left || (kByUnit && i != warp)) continue;
    const CrossRow r = cross_row(c, u.b, u.rho0 + row0 + i);
    const bool some = cross_some(c, r, ll[i]);
    const long long at = cross_out_row(c, r, u.h);
    const float norm = some ? 1.f / ll[i] : 0.f;
    __nv_bfloat16* const to = reinterpret_cast<__nv_bfloat16*>(c.out) + at * kD + kPer * lane;
#pragma unroll
    for (int z = 0; z < kPer; z += 2) reinterpret_cast<uint32_t*>(to)[z / 2] = some ? pack_bf16x2(acc[i][z] * norm, acc[i][z + 1] * norm) : 0u;
    if (lane == 0 && c.lse) c.lse[at] = some ? fmaf(mm[i], 0.6931471805599453f, logf(ll[i])) : -INFINITY;
  }
}

// By units, and by pieces, where a unit is shared by eight CTAs or more.
template <int kD, int kRows>
cudaError_t launch_merge(const CrossProblem& c, const float* part, const int2* begins, int row_tiles, int ctas, cudaStream_t st) {
  const long long units = (long long)c.sources * c.Hkv * row_tiles;
  const bool by_unit = 8 * units <= ctas;
  const unsigned int x = (unsigned int)(by_unit ? units : ctas), rows = (unsigned int)(c.rows() < kRows ? c.rows() : kRows);
  constexpr int kAtOnce = kRows <= 32 ? 1 : 2, kBlock = 8 * kAtOnce;
  if (by_unit) return launch_chained(cross_merge_kernel<kD, kRows, kAtOnce, 4, true>, dim3(x, (rows + kAtOnce - 1) / kAtOnce), 256, 0, st, c, part, begins, ctas, row_tiles);
  return launch_chained(cross_merge_kernel<kD, kRows, kAtOnce, 2, false>, dim3(x, (rows + kBlock - 1) / kBlock), 256, 0, st, c, part, begins, ctas, row_tiles);
}

}  // namespace
}  // namespace restkv
