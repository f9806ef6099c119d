// Cross attention of few query rows of a KV head (hypotheses x tokens x heads of the group) on the warp-level tensor instructions: bf16,
// head_dim 64 or 128.
//
// What bounds it: K and V are read once, for all hypotheses of a source, and meet up to 32 query rows per pass: the step streams HBM.
//   - a warp owns every eighth (fourth) tile of its CTA's run and a ring of tile slots that its own lane fills by TMA from K and V as they lie (four
//     dimensions with strides; 128-byte swizzle for ldmatrix), so that warps never wait for one another while they stream;
//   - mma.sync m16n8k16 with rows of the cache as rows, query rows as columns: S^T = K Q^T, O^T = V^T P^T.  Tiles of 8 query rows, 1, 2 or 4
//     of them, so that few rows are not padded and 32 read K and V once; of 32 the queries are read from shared memory, where O has the registers;
//   - weights as two bf16 parts (16 bits): the tensor pipe has room for the second product beside HBM.
// Work is split as in the attention over pages: a cluster of CTAs per unit (source, KV head, query rows) for short sources, merged through
// distributed shared memory in one launch; the tiles of all units end to end, an even share of them per CTA, and a second kernel that joins
// what several CTAs left of a unit, for long ones and for batches of any lengths.
#include <math.h>

#include <type_traits>

#include <cooperative_groups.h>

#include "cross_tc.cuh"
#include "paged_deal.cuh"
#include "warp_mma.cuh"

namespace restkv {

namespace {

namespace cg = cooperative_groups;

constexpr int kFewSnap = 8;                     // tiles that a CTA could go through while it ends one unit and begins another
constexpr float kFewSlack = 8.f;                // log2 of what weights may grow to before O is rescaled

struct CrossFewArgs {
  CrossProblem c;
  float* part;                                  // per CTA two of: o [rows, d], (m, l) [rows]; without clusters
  int2* begins;                                 // per CTA: unit and tile of it that it begins with; -1: none
  unsigned int* dev_status;
  int row_tiles;                                // units per KV head
  int cluster;                                  // CTAs per unit, 0: tiles of all units end to end
  long long wait_limit;
};

template <int kD, int kNT, bool kCluster> struct FewConfig {
  // Dealt out, two CTAs of four warps share an SM: one streams while the other ends a unit and begins the next.
  static constexpr int kWarps = kCluster ? 8 : 4, kThreads = kWarps * 32, kPerSm = kCluster ? 1 : 2;
  static constexpr int kRows = 8 * kNT;
  static constexpr int kBlocks = kD == 64 ? 2 : 1;                        // blocks of 16 rows of a tile
  static constexpr int kTileRows = 16 * kBlocks;
  static constexpr uint32_t kBox = kTileRows * 128;                       // [rows x 64 dims]
  static constexpr uint32_t kSide = kTileRows * kD * 2;                   // K's, or V's
  static constexpr uint32_t kStageBytes = 2 * kSide;
  static constexpr int kStages = kCluster ? 2 : 3;
  static constexpr bool kQInShared = kNT > 2;
  static constexpr uint32_t kQBytes = kQInShared ? kRows * kD * 2u : 0u;
  static constexpr uint32_t kPartBytes = kRows * kD * 4u;                 // a warp's o in the merge
  static constexpr uint32_t kPushBytes = kCluster ? kPartBytes + 256u + 16u * kRows * 8u : 0u;   // what the peers push
  static constexpr size_t kSmem = (size_t)kWarps * kStages * kStageBytes + kQBytes + kPushBytes + 1024;
  static_assert(kStages * kStageBytes >= kPartBytes, "the merge needs the ring's space");
};

__device__ __forceinline__ int few_entries(const CrossProblem& c) { return c.per_head ? c.sources * c.Hkv : c.sources; }
__device__ __forceinline__ int few_units(const CrossProblem& c, int row_tiles) { return c.per_head ? row_tiles : c.Hkv * row_tiles; }
__device__ __forceinline__ int few_tiles(const CrossProblem& c, int entry, int tile_rows) {
  const int n = c.per_head ? cross_length(c, entry / c.Hkv, entry % c.Hkv) : cross_length(c, entry, 0);
  const int t = (n + tile_rows - 1) / tile_rows;
  return t > 0 ? t : 1;                         // a unit without rows has its outputs written, too
}

// Dims 4 v .. of a query row's result.
template <int kD> __device__ __forceinline__ void few_write(const CrossProblem& c, int source, int h, int rho, int v, float4 acc, float mm, float ll) {
  const CrossRow r = cross_row(c, source, rho);
  const bool some = cross_some(c, r, ll);
  const long long at = cross_out_row(c, r, h);
  const float f = some ? 1.f / ll : 0.f;
  reinterpret_cast<uint2*>(reinterpret_cast<__nv_bfloat16*>(c.out) + at * kD)[v] =
      some ? make_uint2(pack_bf16x2(acc.x * f, acc.y * f), pack_bf16x2(acc.z * f, acc.w * f)) : make_uint2(0u, 0u);
  if (v == 0 && c.lse) c.lse[at] = some ? fmaf(mm, 0.6931471805599453f, logf(ll)) : -INFINITY;
}

template <int kD, int kNT, bool kCluster>
__global__ void __launch_bounds__(FewConfig<kD, kNT, kCluster>::kThreads, FewConfig<kD, kNT, kCluster>::kPerSm)
cross_few_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const __grid_constant__ CrossFewArgs a) {
  using C = FewConfig<kD, kNT, kCluster>;
  constexpr int kRows = C::kRows, kBlocks = C::kBlocks, kW = C::kWarps, kStages = C::kStages, kThreads = C::kThreads;
  constexpr uint32_t ring_bytes = (uint32_t)kStages * C::kStageBytes;
  const CrossProblem& c = a.c;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t full[kW][kStages];
  __shared__ float w_ml[kW][kRows][2];
  __shared__ float w_factor[kW][kRows];
  __shared__ float2 c_ml[kRows];
  __shared__ float push_factor[kCluster ? 16 : 1][kRows];
  __shared__ int abort_flag;
  __shared__ Piece piece_s;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, r = lane >> 2, q4 = lane & 3, mat = lane >> 3, mr = lane & 7;
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* rings = smem_raw + (smem_base - smem_u32(smem_raw));
  uint8_t* ring = rings + warp * ring_bytes;
  const uint32_t ring_addr = smem_base + (uint32_t)warp * ring_bytes, q_addr = smem_base + kW * ring_bytes;
  uint8_t* const push = rings + kW * ring_bytes + C::kQBytes;
  const int R = (int)c.rows();

  if (threadIdx.x == 0) abort_flag = 0;
  if (lane == 0) {
    for (int s = 0; s < kStages; ++s) mbar_init(&full[warp][s], 1);
    fence_mbar_init();
    prefetch_tensormap(&tmK);
    prefetch_tensormap(&tmV);
  }
  __syncwarp();
  if (kCluster) cluster_arrive();               // peers push into shared memory once all have begun
  grid_dependency_wait();
  grid_dependency_launch();

  auto tiles_of = [&](int entry) { return few_tiles(c, entry, C::kTileRows); };
  if constexpr (!kCluster) {
    if (warp == 0) {
      const Run run = find_run(few_entries(c), few_units(c, a.row_tiles), tiles_of, kFewSnap, blockIdx.x, gridDim.x);
      if (lane == 0) {
        piece_s.run = run;
        if (run.tile < run.end) piece_s.cut(few_units(c, a.row_tiles), tiles_of);
        a.begins[blockIdx.x] = run.tile < run.end ? make_int2(piece_s.unit, piece_s.t0) : make_int2(-1, 0);
      }
    }
    __syncthreads();
    if (piece_s.run.tile >= piece_s.run.end) return;
  } else {
    __syncthreads();
  }

  int slot = 0;                                 // of the warp's ring: the next tile's, and the parity it completes with
  uint32_t parity = 0;
  for (;;) {
    bool ok = true;                             // false: a wait ran out
    const volatile Piece& piece = piece_s;
    const int unit = kCluster ? (int)(blockIdx.x / (unsigned int)a.cluster) : piece.unit;
    const int bh = unit / a.row_tiles, rho0 = (unit - bh * a.row_tiles) * kRows, b = bh / c.Hkv, h = bh - b * c.Hkv;
    // the warp's tiles: `stride` apart from `next` on, below t1
    const int cluster_rank = kCluster ? (int)(blockIdx.x % (unsigned int)a.cluster) : 0, stride = kCluster ? a.cluster * kW : kW;
    const int next = (kCluster ? cluster_rank * kW : piece.t0) + warp;
    auto tiles_below = [&](int t1) { return t1 > next ? (t1 - next + stride - 1) / stride : 0; };
    auto request = [&](int i, int s) {          // tile i into slot s, by one lane
      uint8_t* dst = ring + (uint32_t)s * C::kStageBytes;
      uint64_t* bar = &full[warp][s];
      const int row = (next + i * stride) * C::kTileRows;
      mbar_arrive_expect_tx(bar, C::kStageBytes);
#pragma unroll
      for (int x = 0; x < kD / 64; ++x) {
        tma_load_4d(dst + x * C::kBox, &tmK, bar, x * 64, row, h, b);
        tma_load_4d(dst + C::kSide + x * C::kBox, &tmV, bar, x * 64, row, h, b);
      }
    };
    // in clusters the first tiles are asked for before the source's length is known: as many as K and V have
    int asked = 0;
    if (kCluster) {
      asked = min(tiles_below((c.n_rows + C::kTileRows - 1) / C::kTileRows), kStages);
      if (elect_one()) {
        for (int i = 0; i < asked; ++i) request(i, i);
      }
    }
    const int n = cross_length(c, b, h), n_tiles = (n + C::kTileRows - 1) / C::kTileRows;
    const int mine = tiles_below(kCluster ? n_tiles : min(piece.t1, n_tiles));
    if (!kCluster && elect_one()) {
      for (int i = 0; i < kStages && i < mine; ++i) request(i, slot + i < kStages ? slot + i : slot + i - kStages);
    }
    __syncwarp();

    // ---- the query rows as the B operand ----
    uint32_t qb[C::kQInShared ? 1 : kD / 16][C::kQInShared ? 1 : kNT][2];
    if constexpr (C::kQInShared) {
      constexpr int kChunks = kD / 8;
      for (int x = threadIdx.x; x < kRows * kChunks; x += kThreads) {
        const int row = x / kChunks, chunk = x % kChunks, rho = rho0 + row;
        uint4 u = make_uint4(0u, 0u, 0u, 0u);
        if (rho < R) u = reinterpret_cast<const uint4*>(cross_query<__nv_bfloat16>(c, cross_row(c, b, rho), h))[chunk];
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(q_addr + (uint32_t)row * (kD * 2) + (uint32_t)((chunk ^ (row & 7)) << 4)), "r"(u.x), "r"(u.y), "r"(u.z),
                     "r"(u.w) : "memory");
      }
      __syncthreads();
    } else {
#pragma unroll
      for (int t = 0; t < kNT; ++t) {
        const int rho = rho0 + r + 8 * t;
        const bool live = rho < R;
        const uint32_t* q = reinterpret_cast<const uint32_t*>(cross_query<__nv_bfloat16>(c, cross_row(c, b, live ? rho : 0), h));
#pragma unroll
        for (int k = 0; k < kD / 16; ++k) {
          qb[k][t][0] = live ? q[8 * k + q4] : 0u;
          qb[k][t][1] = live ? q[8 * k + 4 + q4] : 0u;
        }
      }
    }
    auto for_queries = [&](int k, auto&& use) { // step k's operand of every tile of query rows
      if constexpr (C::kQInShared) {
#pragma unroll
        for (int t = 0; t < kNT; t += 2) {
          uint32_t w[4];
          ldsm4(q_addr + (uint32_t)(8 * t + (mat >> 1) * 8 + mr) * (kD * 2) + (uint32_t)(((2 * k + (mat & 1)) ^ mr) << 4), w);
          use(t, w[0], w[1]);
          use(t + 1, w[2], w[3]);
        }
      } else {
#pragma unroll
        for (int t = 0; t < kNT; ++t) use(t, qb[k][t][0], qb[k][t][1]);
      }
    };

    const float factor = c.scale * kLog2e;
    float ref[kNT][2], l[kNT][2], o[kD / 16][kNT][4];
#pragma unroll
    for (int t = 0; t < kNT; ++t) {
      ref[t][0] = ref[t][1] = -INFINITY;
      l[t][0] = l[t][1] = 0.f;
#pragma unroll
      for (int x = 0; x < kD / 16; ++x) o[x][t][0] = o[x][t][1] = o[x][t][2] = o[x][t][3] = 0.f;
    }
    auto take = [&](auto edge, uint32_t stage, int row0) {
      constexpr bool kEdge = decltype(edge)::value;
      float sc[kBlocks][kNT][4];
#pragma unroll
      for (int k = 0; k < kBlocks; ++k) {
#pragma unroll
        for (int t = 0; t < kNT; ++t) sc[k][t][0] = sc[k][t][1] = sc[k][t][2] = sc[k][t][3] = 0.f;
#pragma unroll
        for (int x = 0; x < kD / 16; ++x) {
          uint32_t w[4];
          ldsm4(stage + (uint32_t)(x >> 2) * C::kBox + (uint32_t)(k * 16 + (mat & 1) * 8 + mr) * 128u + (((uint32_t)((x & 3) * 2 + (mat >> 1)) ^ (uint32_t)mr) << 4), w);
          for_queries(x, [&](int t, uint32_t b0, uint32_t b1) { mma16816(sc[k][t], w, b0, b1); });
        }
#pragma unroll
        for (int t = 0; t < kNT; ++t)
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            sc[k][t][x] *= factor;
            if (kEdge && row0 + 16 * k + r + 8 * (x >> 1) >= n) sc[k][t][x] = -INFINITY;
          }
      }
      float f[kNT][2];
      bool grown = false;
#pragma unroll
      for (int t = 0; t < kNT; ++t)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float mx = fmaxf(sc[0][t][e], sc[0][t][2 + e]);
#pragma unroll
          for (int k = 1; k < kBlocks; ++k) mx = fmax3(mx, sc[k][t][e], sc[k][t][2 + e]);
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
          f[t][e] = 1.f;
          if (mx > ref[t][e] + kFewSlack) {     // o is rescaled only when the weights would grow past 2^kFewSlack
            f[t][e] = ex2_approx(ref[t][e] - mx);   // ref = -inf gives 0
            ref[t][e] = mx;
            l[t][e] *= f[t][e];
            grown = true;
          }
          const float m_use = ref[t][e] == -INFINITY ? 0.f : ref[t][e];   // only logits of -inf so far: they weigh nothing
#pragma unroll
          for (int k = 0; k < kBlocks; ++k) {
            sc[k][t][e] = ex2_approx(sc[k][t][e] - m_use);
            sc[k][t][2 + e] = ex2_approx(sc[k][t][2 + e] - m_use);
            l[t][e] += sc[k][t][e] + sc[k][t][2 + e];
          }
        }
      if (__any_sync(0xffffffffu, grown)) {
#pragma unroll
        for (int t = 0; t < kNT; ++t)
#pragma unroll
          for (int x = 0; x < kD / 16; ++x)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[x][t][e] *= f[t][e & 1];
      }
#pragma unroll
      for (int k = 0; k < kBlocks; ++k) {
        // bits of the rows 2 q4, 2 q4 + 1 (+ 8) of V that are there: past them is anything, and a weight of 0 is to find a number
        uint32_t keep0 = 0xFFFFFFFFu, keep1 = 0xFFFFFFFFu;
        if constexpr (kEdge) {
          const int left = n - (row0 + 16 * k) - 2 * q4;
          keep0 = (left > 0 ? 0xFFFFu : 0u) | (left > 1 ? 0xFFFF0000u : 0u);
          keep1 = (left > 8 ? 0xFFFFu : 0u) | (left > 9 ? 0xFFFF0000u : 0u);
        }
        uint32_t pb[kNT][4];                    // the upper parts of the weights, then what they leave
#pragma unroll
        for (int t = 0; t < kNT; ++t)
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const float p0 = sc[k][t][2 * x], p1 = sc[k][t][2 * x + 1];
            const uint32_t hi = pack_bf16x2(p0, p1);
            pb[t][x] = transpose8x8(hi);
            pb[t][2 + x] = transpose8x8(pack_bf16x2(p0 - lower(hi), p1 - upper(hi)));
          }
#pragma unroll
        for (int x = 0; x < kD / 16; ++x) {
          uint32_t va[4];
          ldsm4_t(stage + C::kSide + (uint32_t)(x >> 2) * C::kBox + (uint32_t)(k * 16 + (mat >> 1) * 8 + mr) * 128u + (((uint32_t)((x & 3) * 2 + (mat & 1)) ^ (uint32_t)mr) << 4), va);
          if constexpr (kEdge) { va[0] &= keep0; va[1] &= keep0; va[2] &= keep1; va[3] &= keep1; }
#pragma unroll
          for (int t = 0; t < kNT; ++t) {
            mma16816(o[x][t], va, pb[t][0], pb[t][1]);
            mma16816(o[x][t], va, pb[t][2], pb[t][3]);
          }
        }
      }
    };

    for (int i = 0; i < mine; ++i) {
      ok = __all_sync(0xffffffffu, mbar_wait_within(&full[warp][slot], parity, &abort_flag, a.dev_status, kDevTimeout, a.wait_limit));
      if (!ok) {
        if (lane == 0)                          // nothing may still be on its way into shared memory when the CTA returns
          for (int j = 0; j < kStages && i + j < max(mine, asked); ++j) {
            const int s = slot + j < kStages ? slot + j : slot + j - kStages;
            wait_issued(&full[warp][s], s < slot ? parity ^ 1u : parity);
          }
        break;
      }
      const uint32_t stage = ring_addr + (uint32_t)slot * C::kStageBytes;
      const int row0 = (next + i * stride) * C::kTileRows;
      if (row0 + C::kTileRows > n) take(std::true_type{}, stage, row0);
      else take(std::false_type{}, stage, row0);
      __syncwarp();                             // every lane has read the slot
      if (i + kStages < mine && elect_one()) request(i + kStages, slot);
      __syncwarp();
      if (++slot == kStages) { slot = 0; parity ^= 1u; }
    }

    // (tiles past the source's rows: they have to be there before their places serve for something else)
    if (kCluster && ok)
      for (int i = mine; i < asked; ++i) wait_issued(&full[warp][i % kStages], (uint32_t)(i / kStages));

    // ---- merge, in a fixed order: the warps of the CTA through their (idle) rings ----
    __syncwarp();
    // [rows][kD / 4] float4, a row's order such that the four rows that lanes store side by side go to different banks
    auto w_o = [&](int w, int row, int v) { return reinterpret_cast<float4*>(rings + w * ring_bytes) + row * (kD / 4) + (v ^ ((row >> 1 & 3) << 1)); };
#pragma unroll
    for (int t = 0; t < kNT; ++t) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float x = l[t][e];
        x += __shfl_xor_sync(0xffffffffu, x, 4);
        x += __shfl_xor_sync(0xffffffffu, x, 8);
        x += __shfl_xor_sync(0xffffffffu, x, 16);
        if (r == 0) { w_ml[warp][2 * q4 + e + 8 * t][0] = ref[t][e]; w_ml[warp][2 * q4 + e + 8 * t][1] = x; }
      }
      if (mine > 0) {
#pragma unroll
        for (int x = 0; x < kD / 16; ++x)       // dims 16 x + r, 16 x + 8 + r
#pragma unroll
          for (int e = 0; e < 4; ++e) reinterpret_cast<float*>(w_o(warp, 2 * q4 + 8 * t + (e & 1), 4 * x + 2 * (e >> 1) + (r >> 2)))[r & 3] = o[x][t][e];
      }
    }
    __syncthreads();
    const int rows = R - rho0 < kRows ? R - rho0 : kRows;
    for (int x = threadIdx.x; x < kRows * kW; x += kThreads) {   // a warp's factor for each row, and the CTA's (reference, sum)
      const int row = x / kW, w = x % kW;
      const float mw = w_ml[w][row][0];
      float mm = mw;
#pragma unroll
      for (int off = kW / 2; off > 0; off >>= 1) mm = fmaxf(mm, __shfl_xor_sync(0xffffffffu, mm, off));
      const float f = mw == -INFINITY ? 0.f : ex2_approx(mw - mm);
      float ll = w_ml[w][row][1] * f;
#pragma unroll
      for (int off = kW / 2; off > 0; off >>= 1) ll += __shfl_xor_sync(0xffffffffu, ll, off);
      w_factor[w][row] = f;
      if (w == 0) c_ml[row] = make_float2(mm, ll);
    }
    __syncthreads();
    const int items = rows * (kD / 4);          // four dims of a row
    // of the units that it shares, a CTA has the beginning of one at most and none of that of another: a slot for each
    float* const part = a.part + (long long)(2 * blockIdx.x + (piece.t0 == 0)) * kRows * (kD + 2);
    // in clusters the results of item x are merged by CTA x % cluster
    float2* const push_ml = reinterpret_cast<float2*>(push);                                // [cluster][kRows]
    float4* const push_o = reinterpret_cast<float4*>(push + 16 * kRows * sizeof(float2));   // [cluster][items / cluster, rounded up]
    const int per_cta = kCluster ? (items + a.cluster - 1) / a.cluster : 0;
    const int whole = kCluster ? 0 : piece.whole;
    if (kCluster) cluster_wait();
    for (int x = threadIdx.x; x < items; x += kThreads) {
      const int row = x / (kD / 4), v = x % (kD / 4);
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < kW; ++w) {
        const float f = w_factor[w][row];
        if (f == 0.f) continue;
        fma4(acc, *w_o(w, row, v), f);
      }
      if (kCluster) {
        *cg::this_cluster().map_shared_rank(push_o + cluster_rank * per_cta + x / a.cluster, x % a.cluster) = acc;
      } else if (whole) {
        few_write<kD>(c, b, h, rho0 + row, v, acc, c_ml[row].x, c_ml[row].y);
      } else {
        reinterpret_cast<float4*>(part)[row * (kD / 4) + v] = acc;
        if (v == 0) reinterpret_cast<float2*>(part + kRows * kD)[row] = c_ml[row];
      }
    }
    if constexpr (kCluster) {
      for (int x = threadIdx.x; x < rows * a.cluster; x += kThreads) {
        const int to = x / rows, row = x - to * rows;
        *cg::this_cluster().map_shared_rank(push_ml + cluster_rank * kRows + row, to) = c_ml[row];
      }
      __syncwarp();
      cluster_arrive();
      cluster_wait();
      // the CTAs' factors for each row, a.cluster threads side by side to a row
      for (int x = threadIdx.x; x - (int)(threadIdx.x & 31) < rows * a.cluster; x += kThreads) {   // whole warps stay
        const int row = x / a.cluster, from = x & (a.cluster - 1);
        const float2 ml = row < rows ? push_ml[from * kRows + row] : make_float2(-INFINITY, 0.f);
        float mm = ml.x;
        for (int off = a.cluster / 2; off > 0; off >>= 1) mm = fmaxf(mm, __shfl_xor_sync(0xffffffffu, mm, off));
        const float f = ml.x == -INFINITY ? 0.f : ex2_approx(ml.x - mm);
        float ll = ml.y * f;
        for (int off = a.cluster / 2; off > 0; off >>= 1) ll += __shfl_xor_sync(0xffffffffu, ll, off);
        if (row < rows) {
          push_factor[from][row] = f;
          if (from == 0) c_ml[row] = make_float2(mm, ll);
        }
      }
      __syncthreads();
      for (int y = threadIdx.x; y < per_cta; y += kThreads) {
        const int x = y * a.cluster + cluster_rank;
        if (x >= items) continue;
        const int row = x / (kD / 4);
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int from = 0; from < a.cluster; ++from) fma4(acc, push_o[from * per_cta + y], push_factor[from][row]);
        few_write<kD>(c, b, h, rho0 + row, x % (kD / 4), acc, c_ml[row].x, c_ml[row].y);
      }
      return;
    }
    // all of the CTA's warps go on to the next piece or none
    if (__syncthreads_or(!ok)) return;
    if (threadIdx.x == 0) {
      piece_s.run.tile += piece_s.t1 - piece_s.t0;
      if (piece_s.run.tile < piece_s.run.end) piece_s.cut(few_units(c, a.row_tiles), tiles_of);
    }
    __syncthreads();
    if (piece_s.run.tile >= piece_s.run.end) return;
    fence_proxy_async_smem();                   // the rings were written by ordinary stores; bulk copies come next
  }
}

// ---- host ----
struct FewVariant {
  void (*kernel)(CUtensorMap, CUtensorMap, CrossFewArgs);
  void (*in_clusters)(CUtensorMap, CUtensorMap, CrossFewArgs);
  cudaError_t (*merge)(const CrossProblem&, const float*, const int2*, int, int, cudaStream_t);
  int d, rows, tile_rows, threads, cluster_threads, per_sm;
  size_t smem, cluster_smem;
};
template <int kD, int kNT> FewVariant few_variant() {
  using C = FewConfig<kD, kNT, false>;
  using K = FewConfig<kD, kNT, true>;
  return FewVariant{cross_few_kernel<kD, kNT, false>, cross_few_kernel<kD, kNT, true>, launch_merge<kD, C::kRows>, kD, C::kRows, C::kTileRows, C::kThreads, K::kThreads,
                    C::kPerSm, C::kSmem, K::kSmem};
}
int few_ctas(const FewVariant& v, int sm_count) { return v.per_sm * sm_count < kMaxCtas ? v.per_sm * sm_count : kMaxCtas; }
// Up to 8 query rows in one tile of 8, up to 16 in two; more in four, 32 of them per pass over K and V.
template <int kD> FewVariant few_of(long long rows) { return rows <= 8 ? few_variant<kD, 1>() : rows <= 16 ? few_variant<kD, 2>() : few_variant<kD, 4>(); }
bool pick_few(const CrossProblem& c, long long rows, FewVariant* v) {
  if (c.d != 64 && c.d != 128) return false;
  *v = c.d == 64 ? few_of<64>(rows) : few_of<128>(rows);
  return true;
}

// How a call would run: CTAs per unit of a launch in clusters, 0 for one that deals out the tiles of all units, and about how long, in us.  Fixed 6, and 12 or 16
// (these have another kernel behind them), and the bytes at what HBM and the CTAs draw: by the tiles of query rows, 0.09, 0.07 or 0.044 TB/s each.
// Fitted to the times below and their like, on 148 SMs: dealt out, as much as 118 CTAs draw, 6.1 TB/s at most; in clusters 5.5.  A cluster lasts as long as its own source, so that
// sources of different lengths, which only the device knows, speak for dealing out: 0.8 of the rows are taken to be there.  Measured, 8 KV heads of 128 with 32 query rows,
// 30000 rows: clusters of 4 90.0 us, of 8 50.9, dealt out 36.0; 4000 rows 18.8, 13.9, 17.4; 16 query rows over 1500 rows 8.9, 8.3, 13.0.
struct FewWay {
  int cluster;
  double us;
};
FewWay few_way(const CrossProblem& c, const FewVariant& v, long long units, const int* clusters_of) {
  const double mb = 4e-6 * (double)units * c.n_rows * c.d, each = v.rows == 8 ? 0.09 : v.rows == 16 ? 0.07 : 0.044;
  const double fill = c.lengths && (c.sources > 1 || c.per_head) ? 0.8 : 1.0;
  FewWay best{0, (v.rows == 32 ? 16.0 : 12.0) + fill * mb / fmin(118.0 * each, 6.1)};
  for (int i = 1; i < 5; ++i) {
    if (units > clusters_of[i]) break;
    const double us = 6.0 + mb / fmin(each * (double)(units << i), 5.5);
    if (us < best.us) best = FewWay{1 << i, us};
  }
  return best;
}

}  // namespace

cudaError_t cross_few_init() {
  CrossProblem c{};
  for (int d : {64, 128})
    for (int rows : {8, 16, 32}) {
      c.d = d;
      FewVariant v;
      if (!pick_few(c, rows, &v)) continue;
      cudaError_t e = cudaFuncSetAttribute(v.kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)v.smem);
      if (e == cudaSuccess) e = cudaFuncSetAttribute(v.in_clusters, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)v.cluster_smem);
      if (e == cudaSuccess) e = cudaFuncSetAttribute(v.in_clusters, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
      if (e != cudaSuccess) return e;
    }
  return cudaSuccess;
}

bool cross_few_supported(const CrossProblem& c) {
  FewVariant v;
  if (!pick_few(c, c.rows(), &v) || !cross_map_fits(c, c.K) || !cross_map_fits(c, c.V)) return false;
  const long long units = (long long)c.sources * c.Hkv * ((c.rows() + v.rows - 1) / v.rows);
  return ((long long)c.n_rows / v.tile_rows + 1) * units <= 0x7FFFFFFFll;   // tiles are counted in 32 bits
}

double cross_few_us(const CrossProblem& c, const int* clusters_of) {
  FewVariant v;
  if (!pick_few(c, c.rows(), &v)) return INFINITY;
  return few_way(c, v, (long long)c.sources * c.Hkv * ((c.rows() + v.rows - 1) / v.rows), clusters_of).us;
}

size_t cross_few_bytes(const CrossProblem& c, int sm_count) {
  FewVariant v;
  if (!pick_few(c, c.rows(), &v)) return 0;
  return (size_t)few_ctas(v, sm_count) * (2 * v.rows * (v.d + 2) * sizeof(float) + sizeof(int2));
}

cudaError_t launch_cross_few(void* state, const CrossProblem& c, float* part, int sm_count, const int* clusters_of, long long wait_limit, unsigned int* dev_status,
                             cudaStream_t st, int* launches) {
  FewVariant v;
  if (!pick_few(c, c.rows(), &v)) return cudaErrorInvalidValue;
  CUtensorMap tmK, tmV;
  if (!make_cross_map((TcState*)state, &tmK, c, c.K, (cuuint32_t)v.tile_rows) || !make_cross_map((TcState*)state, &tmV, c, c.V, (cuuint32_t)v.tile_rows)) return cudaErrorInvalidValue;
  CrossFewArgs a{};
  a.c = c; a.part = part; a.dev_status = dev_status; a.wait_limit = wait_limit;
  a.row_tiles = (int)((c.rows() + v.rows - 1) / v.rows);
  const long long units = (long long)c.sources * c.Hkv * a.row_tiles;
  a.cluster = few_way(c, v, units, clusters_of).cluster;
  *launches = 1;
  if (a.cluster) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned int)(units * a.cluster));
    cfg.blockDim = dim3((unsigned int)v.cluster_threads);
    cfg.dynamicSmemBytes = v.cluster_smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned int)a.cluster;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, v.in_clusters, tmK, tmV, a);
  }
  const int ctas = few_ctas(v, sm_count);
  a.begins = reinterpret_cast<int2*>(part + (size_t)2 * ctas * v.rows * (v.d + 2));
  const cudaError_t e = launch_chained(v.kernel, dim3((unsigned int)ctas), v.threads, v.smem, st, tmK, tmV, a);
  if (e != cudaSuccess) return e;
  *launches = 2;
  return v.merge(c, part, a.begins, a.row_tiles, ctas, st);
}

}  // namespace restkv
