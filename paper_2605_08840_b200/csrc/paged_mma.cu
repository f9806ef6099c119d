// Attention of a few query tokens over the paged cache: bf16 in and out, pages of bf16 or of 4-bit codes, head_dim 64, 128 or 256.
//
// What bounds it: every row is read once and meets few query rows (tokens x query heads of a KV head, up to 16 per pass), so the step
// streams HBM; in 4 bits the instructions that turn codes into operands come close behind.  The design follows from that:
//   - warps that never wait for one another while they stream: each owns every kWarps-th tile of its CTA's run and a ring of tile
//     slots that its own lane 0 fills with bulk copies (4 bits: a block of 16 rows lies in one piece, codes and parameters) or TMA
//     boxes (bf16: 128-byte swizzle for ldmatrix);
//   - mma.sync m16n8k16: S^T = K Q^T with 16 cache rows as rows and 8 query rows as columns, O^T = V^T P^T with 16 dims as rows.  Up to 8
//     query rows cost no padding; the weights get from one layout to the other by a transposition of 8 x 8 blocks in registers;
//   - 4-bit rows are laid out for the fragments: a lane's 4 bytes of K are 8 codes of the dims that its operand registers take, its 2
//     bytes of V 4 dims of one row.
//     A code is an operand as it stands: 16 bits x < 1024 are the f16 subnormal 2^-24 x, so that a nibble in the lowest or in the next
//     four bits is 2^-24 or 2^-20 times its code, and products with it are exact in the fp32 accumulator: a shift and four logic
//     operations make 4 operand registers of 8 codes of K.  For V, whose sums over the upper codes of bytes may as well come out of
//     those over whole bytes (upper = (byte - lower) / 16), it is one less.  q is f16 scaled by a
//     power of two per query row (exact down to 2^-28 of the row's largest element).  s = step * (q . code) + offset * sum(q) per
//     group, o = sum f16(p step) code + sum p offset, all sums in fp32.  Every other row of V counts down from its group's top instead,
//     f16(-p step) (15 - code) + p (offset + 15 step): the tensor pipe cuts each product off at the last place of the running sum, and sums of
//     one sign, which the offsets nearly cancel in the end, would keep that (error before the output's rounding 5.3e-3 at 524288 rows of 8 KV
//     heads and 1.7e-2 at 1048576, for 6e-4 at any length; 2% more time).
//     (bf16 16 + code: two operations per register, and the weights' rounding weighs twice as much unless 8 is taken off the codes:
//     60 us for 131072 rows.  e4m3 codes: m16n8k32 is carried out as conversions and f16 products here, 60 us, too.)
// Measured, 32 query heads of 128 over 8 KV heads: 131072 rows of 4 bits 41 us (3.7 TB/s), of bf16 93 us (5.8 TB/s); 2085 rows of 4 bits 8.1 us.
// Work is split in one of two ways:
//   - a cluster of CTAs per unit (sequence, KV head, up to 16 query rows), merged through distributed shared memory: one launch, for
//     short caches, where latency counts;
//   - the tiles of all units end to end, an equal share of them per CTA whatever the sequences' lengths, partial results in the
//     workspace and a second kernel that merges them.  (The last CTA of a unit to arrive at a counter merging them instead: 4 us more at
//     131072 rows, where one CTA reads what 37 left; at 8 x 2176 rows 3 us more.)
#include <math.h>

#include <type_traits>

#include <cooperative_groups.h>
#include <cuda_fp16.h>

#include "paged_deal.cuh"

namespace restkv {

namespace {

namespace cg = cooperative_groups;

constexpr int kSnap = 24;   // a CTA that ends one unit and begins another pays 5 us for it: some 24 tiles

__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t* r) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t addr, uint32_t* r) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma16816(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma16816_f16(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma16816_f16_start(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {   // c = A B
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
               : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {   // of 16-bit elements, a row per four lanes
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ float lg2_approx(float x) {
  float y;
  asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t lds32(uint32_t addr) {
  uint32_t v;
  asm volatile("ld.shared.b32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t addr) {
  uint2 v;
  asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(addr) : "memory");
  return v;
}
// kWords consecutive words of shared memory, aligned to as much as is read at once.
template <int kWords> __device__ __forceinline__ void lds_words(uint32_t addr, uint32_t* w) {
  if constexpr (kWords == 1) {
    w[0] = lds32(addr);
  } else if constexpr (kWords == 2) {
    const uint2 v = lds64(addr);
    w[0] = v.x; w[1] = v.y;
  } else {
#pragma unroll
    for (int i = 0; i < kWords; i += 4) {
      const uint4 v = lds128(addr + 4 * i);
      w[i] = v.x; w[i + 1] = v.y; w[i + 2] = v.z; w[i + 3] = v.w;
    }
  }
}
// The codes at 4 i of both halves of a word as a pair of f16 subnormals: 2^-24 code for even i, 2^-20 code for odd i.
template <int i> __device__ __forceinline__ uint32_t code_pair(uint32_t w) {
  return (i >= 2 ? w >> 8 : w) & (i & 1 ? 0x00F000F0u : 0x000F000Fu);
}

// The shape of an instantiation.  kD head_dim, kGroups groups of a 4-bit row (0: bf16), kNT tiles of 8 query rows.
template <int kD, int kGroups, int kNT> struct Config {
  static constexpr bool kInt4 = kGroups > 0;
  static constexpr int kRows = 8 * kNT;
  // log2 of the largest weight that a rescaling leaves, and of what it may grow to before the next one (in 4 bits times the step, in f16)
  static constexpr float kStart = kInt4 ? 5.f : 0.f, kSlack = kInt4 ? 13.f : 8.f;
  static constexpr uint32_t kBlockBytes = kInt4 ? 8u * kD + 64u * kGroups : 32u * kD;   // 16 rows of K, or of V
  // tiles of two blocks spread the softmax's exchanges and the waits over more rows; at 8 KB and more they cost ring slots
  static constexpr int kBlocks = kBlockBytes <= 2560 ? 2 : 1;
  static constexpr int kTileRows = kBlocks * kBlockRows;
  static constexpr uint32_t kStageBytes = 2 * kBlocks * kBlockBytes;
  static constexpr int kWarps = !kInt4 && kD == 256 ? 4 : 8;
  // two CTAs per SM where 128 registers are enough: one streams while the other merges
  static constexpr int kPerSm = kInt4 && kNT == 1 && kD <= 128 ? 2 : 1;
  static constexpr int kFit = (int)((kPerSm == 2 ? 110u * 1024u : 220u * 1024u) / (kWarps * kStageBytes));
  static constexpr int kStages = kFit < 2 ? 2 : kFit > 6 ? 6 : kFit;
  static constexpr uint32_t kRing = kStages * kStageBytes;
  static constexpr uint32_t kPartBytes = kRows * kD * 4u;                               // a warp's o in the merge
  static constexpr size_t kSmem = (size_t)kWarps * kRing + 1024;
  // in clusters: two slots per warp, and what the peers push
  static constexpr uint32_t kPushBytes = kRows * kD * 4u + 256u + 16u * kRows * 8u;
  static constexpr size_t kClusterSmem = (size_t)kWarps * 2 * kStageBytes + kPushBytes + 1024;
  static_assert(2 * kStageBytes >= kPartBytes, "the merge needs the ring's space");
};

template <int kD, int kGroups, int kNT, bool kCluster>
__global__ void __launch_bounds__(Config<kD, kGroups, kNT>::kWarps * 32, Config<kD, kGroups, kNT>::kPerSm)
paged_mma_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const __grid_constant__ PagedMmaArgs a) {
  using C = Config<kD, kGroups, kNT>;
  constexpr bool kInt4 = C::kInt4;
  constexpr int kW = C::kWarps, kStages = C::kStages, kRows = C::kRows, kBlocks = C::kBlocks, kWords = kD / 32;
  constexpr float kStart = C::kStart, kSlack = C::kSlack;
  constexpr int kG = kInt4 ? kGroups : 1;
  constexpr int kPerGroup = kWords / kG;       // 32-dim blocks of a group
  const PagedCache& c = a.c;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t full[kW][kStages];
  __shared__ float w_ml[kW][kRows][2];
  __shared__ float w_factor[kW][kRows];
  __shared__ float2 c_ml[kRows];
  __shared__ int abort_flag;
  __shared__ Piece piece_s;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, r = lane >> 2, q4 = lane & 3;
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* rings = smem_raw + (smem_base - smem_u32(smem_raw));
  constexpr int stages = kCluster ? 2 : kStages;
  constexpr uint32_t ring_bytes = (uint32_t)stages * C::kStageBytes;
  uint8_t* ring = rings + warp * ring_bytes;
  const uint32_t ring_addr = smem_base + (uint32_t)warp * ring_bytes;
  const int R = c.n_tokens * c.G;

  if (threadIdx.x == 0) abort_flag = 0;
  if (lane == 0) {
    for (int s = 0; s < kStages; ++s) mbar_init(&full[warp][s], 1);
    fence_mbar_init();
    if (!kInt4) {
      prefetch_tensormap(&tmK);
      prefetch_tensormap(&tmV);
    }
  }
  __syncwarp();
  if (kCluster) cluster_arrive();             // peers push into shared memory once all have begun
  grid_dependency_wait();
  grid_dependency_launch();

  auto tiles_of = [&](int entry) { return entry_tiles(c, entry, C::kTileRows); };
  if constexpr (!kCluster) {
    if (warp == 0) {
      const Run run = find_run(c, a.row_tiles, C::kTileRows, kSnap, blockIdx.x, gridDim.x);
      if (lane == 0) {
        piece_s.run = run;
        if (run.tile < run.end) piece_s.cut(units_of(c, a.row_tiles), tiles_of);
      }
    }
    __syncthreads();
    if (piece_s.run.tile >= piece_s.run.end) return;
  } else {
    __syncthreads();
  }

  int slot = 0;                                // of the warp's ring: the next tile's, and the parity it completes with
  uint32_t parity = 0;
  for (;;) {
    bool ok = true;                            // false: a wait ran out
    // ---- the unit and the run of its tiles ----
    int next, t1;                              // the warp's first tile; its tiles are `stride` apart and below t1
    int cluster_rank = 0;
    const volatile Piece& piece = piece_s;     // read again where it is needed
    const int stride = kCluster ? a.cluster * kW : kW;
    auto unit_of_cta = [&]() { return kCluster ? (int)(blockIdx.x / (unsigned int)a.cluster) : piece.unit; };
    if (kCluster) {
      // every CTA of the cluster takes tiles all over the unit, so that its warps' first blocks are known before the length is
      cluster_rank = (int)(blockIdx.x % (unsigned int)a.cluster);
      next = cluster_rank * kW + warp;
      t1 = 0;
    } else {
      next = piece.t0 + warp;
      t1 = piece.t1;
    }
    const int unit = unit_of_cta(), bh = unit / a.row_tiles, rho0 = (unit - bh * a.row_tiles) * kRows, b = bh / c.Hkv, h = bh - b * c.Hkv;

    // ---- the places of the warp's blocks, looked up for 32 / kBlocks tiles at a time, a block per lane ----
    int place = -1, block_of_lane;
    const int per_page = c.page_rows / kBlockRows;
    auto look_up = [&](int i) {                // the page is only looked at once everything that is loaded beside it is on its way
      block_of_lane = (next + (i + lane / kBlocks) * stride) * kBlocks + lane % kBlocks;
      const int at = block_of_lane / per_page;
      place = at < c.table_width ? c.table[(long long)b * c.table_width + at] : -1;
    };
    look_up(0);
    const int n = paged_length(c, b, h), count = paged_count(c, b);
    if (kCluster) t1 = (n + C::kTileRows - 1) / C::kTileRows;
    if (threadIdx.x == 0 && (kCluster ? cluster_rank : piece.t0) == 0) check_length(c, b, h);
    const int blocks = (n + kBlockRows - 1) / kBlockRows;
    const int mine = t1 > next ? (t1 - next + stride - 1) / stride : 0;

    // ---- the query rows rho0 + r (and + 8): loaded before the first blocks are asked for, behind which they would have to wait ----
    // bf16: in the order of the A operand.  4 bits: dims 32 m + 8 q4 .. + 7 in words 4 m .. 4 m + 3.
    uint32_t q_raw[kNT][kD / 8];
#pragma unroll
    for (int t = 0; t < kNT; ++t) {
      const int rho = rho0 + r + 8 * t, i = rho / c.G, g = rho - i * c.G;
      const bool live = rho < R;
      const __nv_bfloat16* q = reinterpret_cast<const __nv_bfloat16*>(a.Q.data) + b * a.Q.sb + (long long)(h * c.G + g) * a.Q.sh + i * a.Q.sn;
      if constexpr (kInt4) {
#pragma unroll
        for (int m = 0; m < kWords; ++m) {
          const uint4 u = live ? *reinterpret_cast<const uint4*>(q + 32 * m + 8 * q4) : make_uint4(0u, 0u, 0u, 0u);
          q_raw[t][4 * m] = u.x; q_raw[t][4 * m + 1] = u.y; q_raw[t][4 * m + 2] = u.z; q_raw[t][4 * m + 3] = u.w;
        }
      } else {
#pragma unroll
        for (int k = 0; k < kD / 16; ++k) {
          q_raw[t][2 * k] = live ? *reinterpret_cast<const uint32_t*>(q + 16 * k + 2 * q4) : 0u;
          q_raw[t][2 * k + 1] = live ? *reinterpret_cast<const uint32_t*>(q + 16 * k + 8 + 2 * q4) : 0u;
        }
      }
    }

    constexpr int kAhead = 32 / kBlocks;       // tiles that are looked up at once
    unsigned int side_by_side = 0;             // bit per lane: the tile that begins with its block lies in one piece
    unsigned int absent = 0;                   // bit slot * kBlocks + block: nothing was loaded there
    auto request = [&](int i, int s) {         // tile i into slot s, by the whole warp
      if (i % kAhead == 0) {
        if (i > 0) look_up(i);
        if (block_of_lane / kBlocks >= t1 || block_of_lane >= blocks) {
          place = -1;
        } else if ((unsigned int)place >= (unsigned int)c.n_pages) {
          place = -1;
          atomicOr(c.dev_status, kDevBadIndex);
        } else {
          place = (place * c.Hkv + h) * per_page + block_of_lane % per_page;
        }
        const int after = __shfl_down_sync(0xffffffffu, place, 1);
        side_by_side = __ballot_sync(0xffffffffu, place >= 0 && (kBlocks == 1 || after == place + 1));
      }
      const int of = i % kAhead * kBlocks;
      const int at = __shfl_sync(0xffffffffu, place, of);
      uint8_t* dst = ring + (uint32_t)s * C::kStageBytes;
      uint64_t* bar = &full[warp][s];
      if (side_by_side >> of & 1u) {
        absent &= ~(((1u << kBlocks) - 1u) << (s * kBlocks));
        if (elect_one()) {
          mbar_arrive_expect_tx(bar, C::kStageBytes);
          if constexpr (kInt4) {               // K's blocks, then V's
            bulk_load(dst, c.K + (long long)at * C::kBlockBytes, kBlocks * C::kBlockBytes, bar);
            bulk_load(dst + kBlocks * C::kBlockBytes, c.V + (long long)at * C::kBlockBytes, kBlocks * C::kBlockBytes, bar);
          } else {
#pragma unroll
            for (int k = 0; k < kBlocks; ++k)
#pragma unroll
              for (int x = 0; x < kD / 64; ++x) {
                tma_load_2d(dst + k * C::kBlockBytes + x * 2048, &tmK, bar, x * 64, (at + k) * kBlockRows);
                tma_load_2d(dst + (kBlocks + k) * C::kBlockBytes + x * 2048, &tmV, bar, x * 64, (at + k) * kBlockRows);
              }
          }
        }
      } else {                                 // two pages, or less than a whole tile
        int one[kBlocks], there = 0;
#pragma unroll
        for (int k = 0; k < kBlocks; ++k) {
          one[k] = __shfl_sync(0xffffffffu, place, of + k);
          there += one[k] >= 0;
          const unsigned int bit = 1u << (s * kBlocks + k);
          absent = one[k] >= 0 ? absent & ~bit : absent | bit;
        }
        if (elect_one()) {
          mbar_arrive_expect_tx(bar, (uint32_t)there * 2 * C::kBlockBytes);
#pragma unroll
          for (int k = 0; k < kBlocks; ++k) {
            if (one[k] < 0) continue;
            if constexpr (kInt4) {
              bulk_load(dst + k * C::kBlockBytes, c.K + (long long)one[k] * C::kBlockBytes, C::kBlockBytes, bar);
              bulk_load(dst + (kBlocks + k) * C::kBlockBytes, c.V + (long long)one[k] * C::kBlockBytes, C::kBlockBytes, bar);
            } else {
#pragma unroll
              for (int x = 0; x < kD / 64; ++x) {
                tma_load_2d(dst + k * C::kBlockBytes + x * 2048, &tmK, bar, x * 64, one[k] * kBlockRows);
                tma_load_2d(dst + (kBlocks + k) * C::kBlockBytes + x * 2048, &tmV, bar, x * 64, one[k] * kBlockRows);
              }
            }
          }
        }
      }
      __syncwarp();
    };
#pragma unroll
    for (int i = 0; i < kStages; ++i)
      if (i < mine && i < stages) request(i, slot + i < stages ? slot + i : slot + i - stages);

    // ---- Q^T as the B operand, kD / 16 steps; what the query rows of the lane's columns 2 q4, 2 q4 + 1 see ----
    // 4 bits: in f16, scaled by a power of two per row (and 2^-4 where the codes come 16 times too large); sums of q per group in the
    // codes' and that scale, which the logits' factor takes out again.
    uint32_t qb[kD / 16][kNT][2];
    float q_sum[kNT][kG][2], to_log2[kNT][2];  // to log2 units, or to the cap's
    int sees[kNT][2];
    int sees_least = n;
    const float factor = c.softcap > 0.f ? fminf(c.scale / c.softcap, 0x1p126f) : c.scale * kLog2e;
#pragma unroll
    for (int t = 0; t < kNT; ++t) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int rho = rho0 + 2 * q4 + e + 8 * t, i = rho / c.G;
        sees[t][e] = rho < R && i < count ? n - (count - 1 - i) : n;
        sees_least = min(sees_least, sees[t][e]);
        to_log2[t][e] = factor;
      }
      if constexpr (kInt4) {
        float top = 0.f;
#pragma unroll
        for (int x = 0; x < kD / 8; ++x) top = fmaxf(top, fmaxf(fabsf(lower(q_raw[t][x])), fabsf(upper(q_raw[t][x]))));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        // 2^e top in [2^14, 2^15), for top of 2^-86 .. 2^100; an infinite one makes the row's logits NaN
        int e = 141 - (int)(__float_as_uint(top) >> 23);
        e = e < -100 ? -100 : e > 100 ? 100 : e;
        const float scale = top < INFINITY ? __uint_as_float((uint32_t)(127 + e) << 23) : __uint_as_float(0x7FFFFFFFu);
        const float unscale = fminf(__uint_as_float((uint32_t)(127 + 24 - e) << 23) * factor, 0x1p126f);   // finite: logits of 0 stay 0
        to_log2[t][0] = __shfl_sync(0xffffffffu, unscale, 8 * q4);
        to_log2[t][1] = __shfl_sync(0xffffffffu, unscale, 8 * q4 + 4);
        float sum[kG];
#pragma unroll
        for (int g = 0; g < kG; ++g) sum[g] = 0.f;
#pragma unroll
        for (int m = 0; m < kWords; ++m) {
          float v[8];
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            v[2 * x] = lower(q_raw[t][4 * m + x]) * scale;
            v[2 * x + 1] = upper(q_raw[t][4 * m + x]) * scale;
          }
          // the pairs (i, i + 4) that a word's codes come in
          qb[2 * m][t][0] = pack_f16x2(v[0], v[4]);
          qb[2 * m][t][1] = pack_f16x2(0x1p-4f * v[1], 0x1p-4f * v[5]);
          qb[2 * m + 1][t][0] = pack_f16x2(v[2], v[6]);
          qb[2 * m + 1][t][1] = pack_f16x2(0x1p-4f * v[3], 0x1p-4f * v[7]);
          sum[m / kPerGroup] += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
        }
#pragma unroll
        for (int g = 0; g < kG; ++g) {
          sum[g] += __shfl_xor_sync(0xffffffffu, sum[g], 1);
          sum[g] += __shfl_xor_sync(0xffffffffu, sum[g], 2);
          sum[g] *= 0x1p-24f;
          q_sum[t][g][0] = __shfl_sync(0xffffffffu, sum[g], 8 * q4);
          q_sum[t][g][1] = __shfl_sync(0xffffffffu, sum[g], 8 * q4 + 4);
        }
      } else {
#pragma unroll
        for (int k = 0; k < kD / 16; ++k) {
          qb[k][t][0] = q_raw[t][2 * k];
          qb[k][t][1] = q_raw[t][2 * k + 1];
        }
      }
    }
    sees_least = __reduce_min_sync(0xffffffffu, sees_least);

    const float cap_log2 = c.softcap * kLog2e;
    float ref[kNT][2], l[kNT][2];              // of the lane's columns: weights are 2^(logit - ref); this lane's share of the sum
    float o[kD / 16][kNT][4];                  // dims of the 16-dim tile (r, r + 8), query rows 2 q4, 2 q4 + 1 (+ 8 per tile)
    float lo[kG][kNT][2];                      // 4 bits: this lane's share of sum p offset
#pragma unroll
    for (int t = 0; t < kNT; ++t) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        ref[t][e] = -INFINITY;
        l[t][e] = 0.f;
#pragma unroll
        for (int g = 0; g < kG; ++g) lo[g][t][e] = 0.f;
      }
#pragma unroll
      for (int k = 0; k < kD / 16; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[k][t][e] = 0.f;
    }

    // One tile; kEdge: some of its rows are not there, or not for every query row.
    auto take = [&](auto edge, uint32_t stage, int row0, unsigned int gone) {
      constexpr bool kEdge = decltype(edge)::value;
      // Rows m, m + 8 of S^T are rows of the block: m itself in bf16; in 4 bits m / 2 + 4 (m % 2), so that the k indices 2 q4, 2 q4 + 1,
      // 2 q4 + 8, 2 q4 + 9 of O^T = V^T P^T are the rows q4 + 4 j, whose codes of V lie a warp's load side by side.
      const int own = kInt4 ? (r >> 1) + 4 * (r & 1) : r;
      // sc[.][.][2 i + e]: row own + 8 i, query row 2 q4 + e
      float sc[kBlocks][kNT][4];
      const uint32_t pick = r & 1 ? 0x3244u : 0x1044u;   // one of a pair of bf16 as fp32
#pragma unroll
      for (int k = 0; k < kBlocks; ++k) {
        const uint32_t kt = stage + k * C::kBlockBytes;
        if constexpr (kInt4) {
          uint32_t w[2][kWords];
#pragma unroll
          for (int half = 0; half < 2; ++half) lds_words<kWords>(kt + (uint32_t)(own + 8 * half) * (kD / 2) + q4 * (kD / 8), w[half]);
#pragma unroll
          for (int g = 0; g < kG; ++g) {
            float acc[kNT][4];
#pragma unroll
            for (int x = g * kPerGroup; x < (g + 1) * kPerGroup; ++x) {
              const uint32_t a0[4] = {code_pair<0>(w[0][x]), code_pair<0>(w[1][x]), code_pair<1>(w[0][x]), code_pair<1>(w[1][x])};
              const uint32_t a1[4] = {code_pair<2>(w[0][x]), code_pair<2>(w[1][x]), code_pair<3>(w[0][x]), code_pair<3>(w[1][x])};
#pragma unroll
              for (int t = 0; t < kNT; ++t) {
                if (x == g * kPerGroup) mma16816_f16_start(acc[t], a0, qb[2 * x][t][0], qb[2 * x][t][1]);
                else mma16816_f16(acc[t], a0, qb[2 * x][t][0], qb[2 * x][t][1]);
                mma16816_f16(acc[t], a1, qb[2 * x + 1][t][0], qb[2 * x + 1][t][1]);
              }
            }
            const uint4 u = lds128(kt + 8 * kD + 64 * g + 16 * (r >> 1));
            const float step[2] = {__uint_as_float(__byte_perm(u.x, 0u, pick)), __uint_as_float(__byte_perm(u.y, 0u, pick))};
            const float off[2] = {__uint_as_float(__byte_perm(u.z, 0u, pick)), __uint_as_float(__byte_perm(u.w, 0u, pick))};
#pragma unroll
            for (int t = 0; t < kNT; ++t)
#pragma unroll
              for (int x = 0; x < 4; ++x) {
                const float q = q_sum[t][g][x & 1];
                sc[k][t][x] = fmaf(step[x >> 1], acc[t][x], g == 0 ? off[x >> 1] * q : fmaf(off[x >> 1], q, sc[k][t][x]));
              }
          }
        } else {
#pragma unroll
          for (int t = 0; t < kNT; ++t) sc[k][t][0] = sc[k][t][1] = sc[k][t][2] = sc[k][t][3] = 0.f;
          const int mat = lane >> 3, mr = lane & 7;
#pragma unroll
          for (int x = 0; x < kD / 16; ++x) {
            uint32_t w[4];
            ldsm4(kt + (uint32_t)(x >> 2) * 2048u + (uint32_t)((mat & 1) * 8 + mr) * 128u + (((uint32_t)((x & 3) * 2 + (mat >> 1)) ^ (uint32_t)mr) << 4), w);
#pragma unroll
            for (int t = 0; t < kNT; ++t) mma16816(sc[k][t], w, qb[x][t][0], qb[x][t][1]);
          }
        }
      }
      // logits in log2 units (first as parts of the cap); rows that a query row does not see weigh nothing
#pragma unroll
      for (int k = 0; k < kBlocks; ++k)
#pragma unroll
        for (int t = 0; t < kNT; ++t)
#pragma unroll
          for (int x = 0; x < 4; ++x) sc[k][t][x] *= to_log2[t][x & 1];
      if (cap_log2 > 0.f) {
        float far = 0.f;
#pragma unroll
        for (int k = 0; k < kBlocks; ++k)
#pragma unroll
          for (int t = 0; t < kNT; ++t) far = fmax3(fmax3(far, fabsf(sc[k][t][0]), fabsf(sc[k][t][1])), fabsf(sc[k][t][2]), fabsf(sc[k][t][3]));
        const bool near = __all_sync(0xffffffffu, far <= kTanhNear);
#pragma unroll
        for (int k = 0; k < kBlocks; ++k)
#pragma unroll
          for (int t = 0; t < kNT; ++t)
#pragma unroll
            for (int x = 0; x < 4; x += 2) {
              float *u = &sc[k][t][x], *v = &sc[k][t][x + 1];
              if (near) {
                const f32x2 z = tanh_near(f2_make(*u, *v));
                *u = f2_lo(z);
                *v = f2_hi(z);
              } else {
                tanh_any(*u, *v);
              }
              *u *= cap_log2;
              *v *= cap_log2;
            }
      }
      if constexpr (kEdge) {
#pragma unroll
        for (int k = 0; k < kBlocks; ++k)
#pragma unroll
          for (int t = 0; t < kNT; ++t)
#pragma unroll
            for (int x = 0; x < 4; ++x)
              if (row0 + k * kBlockRows + own + 8 * (x >> 1) >= sees[t][x & 1] || (gone >> k & 1u)) sc[k][t][x] = -INFINITY;
      }
      // 4 bits: p step is to fit f16 whatever the steps are, so that the reference grows with the largest of them, too
      float v_step[kBlocks][kG][2], v_off[kBlocks][kG][2];
      float most = 0.f;
      if constexpr (kInt4) {
        float top = 0x1p-40f;                  // at least: weights stay well within fp32
        const float from_top = r & 1 ? 15.f : 0.f, sign = r & 1 ? -1.f : 1.f;   // rows 4 .. 7 and 12 .. 15 of a block count down
#pragma unroll
        for (int k = 0; k < kBlocks; ++k)
#pragma unroll
          for (int g = 0; g < kG; ++g) {
            const uint4 u = lds128(stage + (kBlocks + k) * C::kBlockBytes + 8 * kD + 64 * g + 16 * (r >> 1));
            v_step[k][g][0] = __uint_as_float(__byte_perm(u.x, 0u, pick));
            v_step[k][g][1] = __uint_as_float(__byte_perm(u.y, 0u, pick));
            v_off[k][g][0] = fmaf(v_step[k][g][0], from_top, __uint_as_float(__byte_perm(u.z, 0u, pick)));
            v_off[k][g][1] = fmaf(v_step[k][g][1], from_top, __uint_as_float(__byte_perm(u.w, 0u, pick)));
            if constexpr (kEdge) {
              // a row past the cache holds anything: a weight of 0 is to find a number there
#pragma unroll
              for (int x = 0; x < 2; ++x)
                if (row0 + k * kBlockRows + own + 8 * x >= n || (gone >> k & 1u)) v_step[k][g][x] = v_off[k][g][x] = 0.f;
            }
            top = fmax3(top, v_step[k][g][0], v_step[k][g][1]);
            v_step[k][g][0] *= sign;
            v_step[k][g][1] *= sign;
          }
        most = lg2_approx(top);
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
          mx += most;
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 4));
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 8));
          mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 16));
          f[t][e] = 1.f;
          if (mx > ref[t][e] + kSlack) {       // o is rescaled only when the weights would grow past 2^kSlack
            f[t][e] = ex2_approx(ref[t][e] - (mx - kStart));   // ref = -inf gives 0
            ref[t][e] = mx - kStart;
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
        for (int t = 0; t < kNT; ++t) {
#pragma unroll
          for (int k = 0; k < kD / 16; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[k][t][e] *= f[t][e & 1];
          if (kInt4) {
#pragma unroll
            for (int g = 0; g < kG; ++g) { lo[g][t][0] *= f[t][0]; lo[g][t][1] *= f[t][1]; }
          }
        }
      }
#pragma unroll
      for (int k = 0; k < kBlocks; ++k) {
        const uint32_t vt = stage + (kBlocks + k) * C::kBlockBytes;
        if constexpr (kInt4) {
          uint32_t w[4][(kWords + 1) / 2];     // the units of rows q4, q4 + 4, q4 + 8, q4 + 12
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            lds_words<kWords / 2>(vt + (uint32_t)(q4 + 4 * j) * (kD / 2) + r * (kD / 16), w[j]);
            if (j & 1) {                       // (15 - code)
#pragma unroll
              for (int x = 0; x < kWords / 2; ++x) w[j][x] = ~w[j][x];
            }
          }
          uint32_t pb[kNT][2];
#pragma unroll
          for (int x = 0; x < kWords; ++x) {
            if (x % kPerGroup == 0) {
              const int g = x / kPerGroup;
              const float *step = v_step[k][g], *off = v_off[k][g];
#pragma unroll
              for (int t = 0; t < kNT; ++t) {
                const float* p = sc[k][t];
                lo[g][t][0] = fmaf(p[0], off[0], fmaf(p[2], off[1], lo[g][t][0]));
                lo[g][t][1] = fmaf(p[1], off[0], fmaf(p[3], off[1], lo[g][t][1]));
                pb[t][0] = transpose8x8(pack_f16x2(p[0] * step[0], p[1] * step[0]));
                pb[t][1] = transpose8x8(pack_f16x2(p[2] * step[1], p[3] * step[1]));
              }
            }
            const uint32_t y0 = __byte_perm(w[0][x >> 1], w[1][x >> 1], x & 1 ? 0x7632 : 0x5410);
            const uint32_t y1 = __byte_perm(w[2][x >> 1], w[3][x >> 1], x & 1 ? 0x7632 : 0x5410);
            // rows r: the dim of the lower code of a byte; rows r + 8: the whole byte, from which the merge takes the upper one's
            const uint32_t w0 = y0 & 0x00FF00FFu, w1 = y1 & 0x00FF00FFu, z0 = __byte_perm(y0, 0u, 0x4341), z1 = __byte_perm(y1, 0u, 0x4341);
            const uint32_t va[4] = {w0 & 0x000F000Fu, w0, w1 & 0x000F000Fu, w1};
            const uint32_t vb[4] = {z0 & 0x000F000Fu, z0, z1 & 0x000F000Fu, z1};
#pragma unroll
            for (int t = 0; t < kNT; ++t) {
              mma16816_f16(o[2 * x][t], va, pb[t][0], pb[t][1]);
              mma16816_f16(o[2 * x + 1][t], vb, pb[t][0], pb[t][1]);
            }
          }
        } else {
          // bits of the rows 2 q4, 2 q4 + 1 (+ 8) of V that are there: past the cache is anything, and a weight of 0 is to find a number
          uint32_t keep0 = 0xFFFFFFFFu, keep1 = 0xFFFFFFFFu;
          if constexpr (kEdge) {
            const int left = (gone >> k & 1u) ? 0 : n - (row0 + k * kBlockRows) - 2 * q4;
            keep0 = (left > 0 ? 0xFFFFu : 0u) | (left > 1 ? 0xFFFF0000u : 0u);
            keep1 = (left > 8 ? 0xFFFFu : 0u) | (left > 9 ? 0xFFFF0000u : 0u);
          }
          // the weights as two bf16 parts: the tensor pipe has room for the second product beside HBM, and the outputs keep 16 bits
          uint32_t pb[kNT][4];
#pragma unroll
          for (int t = 0; t < kNT; ++t)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
              const float p0 = sc[k][t][2 * x], p1 = sc[k][t][2 * x + 1];
              const uint32_t hi = pack_bf16x2(p0, p1);
              pb[t][x] = transpose8x8(hi);
              pb[t][2 + x] = transpose8x8(pack_bf16x2(p0 - lower(hi), p1 - upper(hi)));
            }
          const int mat = lane >> 3, mr = lane & 7;
#pragma unroll
          for (int x = 0; x < kD / 16; ++x) {
            uint32_t va[4];
            ldsm4_t(vt + (uint32_t)(x >> 2) * 2048u + (uint32_t)((mat >> 1) * 8 + mr) * 128u + (((uint32_t)((x & 3) * 2 + (mat & 1)) ^ (uint32_t)mr) << 4), va);
            if constexpr (kEdge) { va[0] &= keep0; va[1] &= keep0; va[2] &= keep1; va[3] &= keep1; }
#pragma unroll
            for (int t = 0; t < kNT; ++t) {
              mma16816(o[x][t], va, pb[t][0], pb[t][1]);
              mma16816(o[x][t], va, pb[t][2], pb[t][3]);
            }
          }
        }
      }
    };

    for (int i = 0; i < mine; ++i) {
      ok = __all_sync(0xffffffffu, mbar_try_wait(&full[warp][slot], parity));
      if (!ok) ok = __all_sync(0xffffffffu, mbar_wait(&full[warp][slot], parity, &abort_flag, c.dev_status, kDevTimeout, a.wait_limit));
      if (!ok) {
        if (lane == 0)   // nothing may still be on its way into shared memory when the CTA returns
          for (int j = 0; j < stages && i + j < mine; ++j) {
            const int s = slot + j < stages ? slot + j : slot + j - stages;
            wait_issued(&full[warp][s], s < slot ? parity ^ 1u : parity);
          }
        break;
      }
      const uint32_t stage = ring_addr + (uint32_t)slot * C::kStageBytes;
      const int row0 = (next + i * stride) * C::kTileRows;
      const unsigned int gone = absent >> (slot * kBlocks) & ((1u << kBlocks) - 1u);
      if (row0 + C::kTileRows > sees_least || gone != 0) take(std::true_type{}, stage, row0, gone);
      else take(std::false_type{}, stage, row0, 0u);
      __syncwarp();   // every lane has read the slot
      if (i + stages < mine) request(i + stages, slot);
      if (++slot == stages) { slot = 0; parity ^= 1u; }
    }

    // ---- merge, in a fixed order: the warps of the CTA through their (idle) rings ----
    __syncwarp();
    // w_o [rows][kD / 4] float4, a row's order such that the four rows that lanes store side by side go to different banks
    auto w_o = [&](int w, int row, int v) {
      return reinterpret_cast<float4*>(rings + w * ring_bytes) + row * (kD / 4) + (v ^ ((row >> 1 & 3) << 1));
    };
#pragma unroll
    for (int t = 0; t < kNT; ++t) {
      auto over_rows = [](float x) {
        x += __shfl_xor_sync(0xffffffffu, x, 4);
        x += __shfl_xor_sync(0xffffffffu, x, 8);
        return x + __shfl_xor_sync(0xffffffffu, x, 16);
      };
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        l[t][e] = over_rows(l[t][e]);
        if (r == 0) { w_ml[warp][2 * q4 + e + 8 * t][0] = ref[t][e]; w_ml[warp][2 * q4 + e + 8 * t][1] = l[t][e]; }
        if (kInt4) {
#pragma unroll
          for (int g = 0; g < kG; ++g) lo[g][t][e] = over_rows(lo[g][t][e]);
        }
      }
      if (mine > 0) {
        const int row = 2 * q4 + 8 * t;
        if constexpr (kInt4) {
#pragma unroll
          for (int x = 0; x < kWords; ++x) {   // dims 32 x + 4 r + (0..3)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const float *u = &o[2 * x][t][e], *v = &o[2 * x + 1][t][e], add = lo[x / kPerGroup][t][e];
              *w_o(warp, row + e, 8 * x + r) = make_float4(fmaf(u[0], 0x1p24f, add), fmaf(u[2] - u[0], 0x1p20f, add), fmaf(v[0], 0x1p24f, add), fmaf(v[2] - v[0], 0x1p20f, add));
            }
          }
        } else {
#pragma unroll
          for (int x = 0; x < kD / 16; ++x) {  // dims 16 x + r, 16 x + 8 + r
#pragma unroll
            for (int e = 0; e < 4; ++e)
              reinterpret_cast<float*>(w_o(warp, row + (e & 1), 4 * x + 2 * (e >> 1) + (r >> 2)))[r & 3] = o[x][t][e];
          }
        }
      }
    }
    __syncthreads();
    const int unit_now = unit_of_cta(), bh_now = unit_now / a.row_tiles, rho_now = (unit_now - bh_now * a.row_tiles) * kRows;
    const int b_now = bh_now / c.Hkv, h_now = bh_now - b_now * c.Hkv, rows = R - rho_now < kRows ? R - rho_now : kRows;
    if (threadIdx.x < kRows * kW) {            // a warp's factor for each row, and the CTA's (reference, sum)
      const int row = threadIdx.x / kW, w = threadIdx.x % kW;
      const float mw = w_ml[w][row][0];
      float mm = mw;
#pragma unroll
      for (int off = kW / 2; off > 0; off >>= 1) mm = fmaxf(mm, __shfl_xor_sync(0xffffffffu, mm, off));
      const float f = mw == -INFINITY ? 0.f : ex2_approx(mw - mm);   // without tiles, or with none that the row sees
      float ll = w_ml[w][row][1] * f;
#pragma unroll
      for (int off = kW / 2; off > 0; off >>= 1) ll += __shfl_xor_sync(0xffffffffu, ll, off);
      w_factor[w][row] = f;
      if (w == 0) c_ml[row] = make_float2(mm, ll);
    }
    __syncthreads();
    const int items = rows * (kD / 4);         // four dims of a row
    // of the units that it shares, a CTA has the beginning of one at most and none of that of another: a slot for each
    float* const part = a.part + (long long)(2 * blockIdx.x + (piece.t0 == 0)) * kRows * (kD + 2);
    // in clusters the results of item x are merged by CTA x % cluster
    uint8_t* const push = rings + kW * ring_bytes;
    float2* const push_ml = reinterpret_cast<float2*>(push);                                // [cluster][kRows]
    float4* const push_o = reinterpret_cast<float4*>(push + 16 * kRows * sizeof(float2));   // [cluster][items / cluster, rounded up]
    const int per_cta = kCluster ? (items + a.cluster - 1) / a.cluster : 0;
    const int whole = kCluster ? 0 : piece.whole, count_now = paged_count(c, b_now);
    if (kCluster) cluster_wait();
    for (int x = threadIdx.x; x < items; x += kW * 32) {
      const int row = x / (kD / 4), v = x % (kD / 4);
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < kW; ++w) {
        const float f = w_factor[w][row];
        if (f == 0.f) continue;
        fma4(acc, *w_o(w, row, v), f);
      }
      if (kCluster) {
        const int to = x % a.cluster;
        *cg::this_cluster().map_shared_rank(push_o + cluster_rank * per_cta + x / a.cluster, to) = acc;
      } else if (whole) {
        write_row<kD>(a, b_now, h_now, rho_now + row, count_now, v, acc, c_ml[row].x, c_ml[row].y);
      } else {
        reinterpret_cast<float4*>(part)[row * (kD / 4) + v] = acc;
        if (v == 0) reinterpret_cast<float2*>(part + kRows * kD)[row] = c_ml[row];
      }
    }
    if constexpr (kCluster) {
      for (int x = threadIdx.x; x < rows * a.cluster; x += kW * 32) {
        const int to = x / rows, row = x - to * rows;
        *cg::this_cluster().map_shared_rank(push_ml + cluster_rank * kRows + row, to) = c_ml[row];
      }
      __syncwarp();
      cluster_arrive();
      cluster_wait();
      // a.cluster threads side by side hold an item's parts
      const int from = threadIdx.x & (a.cluster - 1);
      for (int y = threadIdx.x / a.cluster; y - (int)((threadIdx.x & 31) / a.cluster) < per_cta; y += kW * 32 / a.cluster) {   // whole warps stay
        const int x = y * a.cluster + cluster_rank;
        const bool there = y < per_cta && x < items;
        const int row = there ? x / (kD / 4) : 0, v = x % (kD / 4);
        const float2 ml = push_ml[from * kRows + row];
        float4 acc = there ? push_o[from * per_cta + y] : make_float4(0.f, 0.f, 0.f, 0.f);
        float mm = ml.x;
        for (int off = a.cluster / 2; off > 0; off >>= 1) mm = fmaxf(mm, __shfl_xor_sync(0xffffffffu, mm, off));
        const float f = ml.x == -INFINITY ? 0.f : ex2_approx(ml.x - mm);
        float ll = ml.y * f;
        acc.x *= f; acc.y *= f; acc.z *= f; acc.w *= f;
        for (int off = a.cluster / 2; off > 0; off >>= 1) {
          ll += __shfl_xor_sync(0xffffffffu, ll, off);
          acc.x += __shfl_xor_sync(0xffffffffu, acc.x, off);
          acc.y += __shfl_xor_sync(0xffffffffu, acc.y, off);
          acc.z += __shfl_xor_sync(0xffffffffu, acc.z, off);
          acc.w += __shfl_xor_sync(0xffffffffu, acc.w, off);
        }
        if (there && from == 0) write_row<kD>(a, b_now, h_now, rho_now + row, count_now, v, acc, mm, ll);
      }
      return;
    }
    // all of the CTA's warps go on to the next piece or none
    if (__syncthreads_or(!ok)) return;
    if (threadIdx.x == 0) {
      piece_s.run.tile += piece_s.t1 - piece_s.t0;
      if (piece_s.run.tile < piece_s.run.end) piece_s.cut(units_of(c, a.row_tiles), tiles_of);
    }
    __syncthreads();
    if (piece_s.run.tile >= piece_s.run.end) return;
    fence_proxy_async_smem();   // the rings were written by ordinary stores; bulk copies come next
  }
}

// grid (units, rows), block 2 kD: merges what several CTAs left of a unit, 8 pieces at a time (kD / 4 threads each).
template <int kD, int kRows>
__global__ void __launch_bounds__(2 * kD) paged_mma_combine_kernel(const __grid_constant__ PagedMmaArgs a, int grid, int tile_rows) {
  grid_dependency_wait();
  grid_dependency_launch();
  __shared__ int run_s[2];
  __shared__ float2 ml_s[kMaxCtas];
  __shared__ float4 acc_s[8][kD / 4];
  const PagedCache& c = a.c;
  const int unit = blockIdx.x, row = blockIdx.y, bh = unit / a.row_tiles, rho = (unit - bh * a.row_tiles) * kRows + row;
  if (rho >= c.n_tokens * c.G) return;
  const int units = units_of(c, a.row_tiles), entry = unit / units;
  const int b = bh / c.Hkv, h = bh - b * c.Hkv, lane = threadIdx.x & 31;
  if (threadIdx.x < 32) {
    // where the unit's entry begins, by the same sums as in the kernel before
    int before = 0, all = 0;
    const int entries = entries_of(c);
    for (int e = threadIdx.x; e < entries; e += 32) {
      const int t = entry_tiles(c, e, tile_rows) * units;
      all += t;
      if (e < entry) before += t;
    }
    all = __reduce_add_sync(0xffffffffu, all);
    before = __reduce_add_sync(0xffffffffu, before);
    if (threadIdx.x == 0) { run_s[0] = all; run_s[1] = before; }
  }
  const int tiles = entry_tiles(c, entry, tile_rows), count = paged_count(c, b);
  __syncthreads();
  const Deal deal(run_s[0], grid, kSnap);
  const int u0 = run_s[1] + (unit - entry * units) * tiles;
  const int x0 = deal.first_of(u0, tiles), pieces = deal.last_of(u0, tiles) - x0 + 1;
  if (pieces == 1) return;                     // it was one CTA's: written
  constexpr int kSlot = kRows * (kD + 2);
  auto piece = [&](int x) { return a.part + (2ll * (x0 + x) + (x == 0)) * kSlot; };
  const int sub = threadIdx.x / (kD / 4), v = threadIdx.x % (kD / 4);
  constexpr int kAhead = 5;                    // requested before the factors are known
  float4 o[kAhead];
#pragma unroll
  for (int k = 0; k < kAhead; ++k)
    if (sub + 8 * k < pieces) o[k] = __ldcg(reinterpret_cast<const float4*>(piece(sub + 8 * k) + row * kD) + v);
  for (int x = threadIdx.x; x < pieces; x += 2 * kD) ml_s[x] = __ldcg(reinterpret_cast<const float2*>(piece(x) + kRows * kD) + row);
  __syncthreads();
  float mm = -INFINITY, ll = 0.f;
  for (int x = lane; x < pieces; x += 32) mm = fmaxf(mm, ml_s[x].x);
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) mm = fmaxf(mm, __shfl_xor_sync(0xffffffffu, mm, off));
  auto factor = [&](int x) { return ml_s[x].x == -INFINITY ? 0.f : ex2_approx(ml_s[x].x - mm); };
  for (int x = lane; x < pieces; x += 32) ll = fmaf(ml_s[x].y, factor(x), ll);
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) ll += __shfl_xor_sync(0xffffffffu, ll, off);
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
  for (int k = 0; k < kAhead; ++k)
    if (sub + 8 * k < pieces) fma4(acc, o[k], factor(sub + 8 * k));
  for (int x = sub + 8 * kAhead; x < pieces; x += 8) fma4(acc, __ldcg(reinterpret_cast<const float4*>(piece(x) + row * kD) + v), factor(x));
  acc_s[sub][v] = acc;
  __syncthreads();
  if (sub != 0) return;
#pragma unroll
  for (int k = 1; k < 8; ++k) fma4(acc, acc_s[k][v], 1.f);
  write_row<kD>(a, b, h, rho, count, v, acc, mm, ll);
}

// ---- host: one set of functions per instantiation ----
struct Variant {
  void (*kernel)(CUtensorMap, CUtensorMap, PagedMmaArgs);
  void (*in_clusters)(CUtensorMap, CUtensorMap, PagedMmaArgs);
  void (*combine)(PagedMmaArgs, int, int);
  int d, threads, per_sm, rows, tile_rows;
  size_t smem, cluster_smem;
  long long max_tiles(const PagedCache& c, long long units) const { return (c.capacity() / tile_rows + 1) * units; }
};

template <int kD, int kGroups, int kNT> Variant variant() {
  using C = Config<kD, kGroups, kNT>;
  return Variant{paged_mma_kernel<kD, kGroups, kNT, false>, paged_mma_kernel<kD, kGroups, kNT, true>, paged_mma_combine_kernel<kD, C::kRows>, kD, C::kWarps * 32, C::kPerSm, C::kRows,
                 C::kTileRows, C::kSmem, C::kClusterSmem};
}

template <int kNT> bool pick_nt(const PagedCache& c, Variant* v) {
  const int groups = c.format == RESTKV_PAGES_INT4 ? c.d / c.group : 0;
  switch (c.d * 16 + groups) {
    case 64 * 16 + 0: *v = variant<64, 0, kNT>(); return true;
    case 64 * 16 + 1: *v = variant<64, 1, kNT>(); return true;
    case 64 * 16 + 2: *v = variant<64, 2, kNT>(); return true;
    case 128 * 16 + 0: *v = variant<128, 0, kNT>(); return true;
    case 128 * 16 + 1: *v = variant<128, 1, kNT>(); return true;
    case 128 * 16 + 2: *v = variant<128, 2, kNT>(); return true;
    case 128 * 16 + 4: *v = variant<128, 4, kNT>(); return true;
    case 256 * 16 + 0: *v = variant<256, 0, kNT>(); return true;
    case 256 * 16 + 2: *v = variant<256, 2, kNT>(); return true;
    case 256 * 16 + 4: *v = variant<256, 4, kNT>(); return true;
    case 256 * 16 + 8: *v = variant<256, 8, kNT>(); return true;
    default: return false;
  }
}

// Up to 8 query rows go through in one tile of 8; more in tiles of 16, which read the cache once per 16.
bool pick(const PagedCache& c, Variant* v) {
  return (long long)c.n_tokens * c.G <= 8 ? pick_nt<1>(c, v) : pick_nt<2>(c, v);
}

// CTAs per unit of a launch in clusters, 0 for one that deals out the tiles of all units.  The largest cluster that lets all units run
// at once; then by the time that each way takes at the longest sequences the table can name, in us: fixed 6 and 12 (the second has
// another kernel behind it), and the bytes at what its CTAs draw.  A cluster lasts as long as its own sequence, so that sequences of
// different lengths speak for dealing out: a batch is taken to fill 0.8 of its table.  Measured, 8 KV heads of 4 query heads, clusters
// against dealt out: 4 bits 2176 rows 8.1 / 13.3, 16384 rows 14.1 / 15.1, 32768 rows 22.2 / 20.1, 8 x 2176 rows 11.4 / 18.9, 8 x 16384
// 38.6 / 44.6; bf16 2176 rows 7.4 / 12.4, 32768 rows 30.8 / 34.0, 131072 rows 103.5 / 92.0, 8 x 2176 rows 16.6 / 25.9.
int paged_mma_cluster(const PagedCache& c, const Variant& v, long long units, const int* clusters_of) {
  int i = 4;
  while (i >= 0 && units > clusters_of[i]) --i;
  if (i < 1) return 0;
  const bool int4 = c.format == RESTKV_PAGES_INT4;
  const double mb = 2e-6 * (double)units * ((double)c.capacity() / kBlockRows) * c.block_bytes;
  // TB/s; clusters of 16 CTAs of which two share an SM end up on half of the SMs
  const double together = v.per_sm == 2 ? (i == 4 ? 2.5 : 0.02 * (double)(units << i)) : 0.085 * (double)(units << i);
  const double fill = c.batch == 1 && !c.per_head ? 1.0 : 0.8;
  const double in_clusters = 6.0 + mb / fmin(together, 5.5), dealt = 12.0 + fill * mb / (int4 ? 5.5 : 6.1);
  return in_clusters < dealt ? 1 << i : 0;
}

}  // namespace

// clusters_of[p][i]: clusters of 2^i CTAs that the device holds at once of kernels with p + 1 CTAs per SM.
cudaError_t paged_mma_init(int (*clusters_of)[5]) {
  PagedCache c{};
  for (int d : {64, 128, 256})
    for (int group : {0, 32, 64, 128})
      for (int rows : {1, 16}) {
        if (group > d) continue;
        c.d = d; c.group = group; c.G = rows; c.n_tokens = 1;
        c.format = group ? RESTKV_PAGES_INT4 : RESTKV_PAGES_BF16;
        Variant v;
        if (!pick(c, &v)) continue;
        cudaError_t e = cudaFuncSetAttribute(v.kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)v.smem);
        if (e == cudaSuccess) e = cudaFuncSetAttribute(v.in_clusters, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)v.cluster_smem);
        if (e == cudaSuccess) e = cudaFuncSetAttribute(v.in_clusters, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        if (e != cudaSuccess) return e;
        if (d != 128 || rows != 1 || (group != 0 && group != 64)) continue;
        for (int i = 0; i < 5; ++i) {
          cudaLaunchConfig_t cfg = {};
          cfg.gridDim = dim3(16);
          cfg.blockDim = dim3((unsigned int)v.threads);
          cfg.dynamicSmemBytes = v.cluster_smem;
          cudaLaunchAttribute attr[1];
          attr[0].id = cudaLaunchAttributeClusterDimension;
          attr[0].val.clusterDim.x = 1u << i;
          attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
          cfg.attrs = attr;
          cfg.numAttrs = 1;
          int* held = &clusters_of[v.per_sm - 1][i];
          *held = 0;
          if (cudaOccupancyMaxActiveClusters(held, v.in_clusters, &cfg) != cudaSuccess) {
            (void)cudaGetLastError();   // a size this device does not take: it holds none of them
            *held = 0;
          }
        }
      }
  return cudaSuccess;
}

bool paged_mma_shape(const PagedCache& c) {
  Variant v;
  return pick(c, &v);
}

bool paged_mma_supported(const PagedCache& c) {
  Variant v;
  if (!pick(c, &v)) return false;
  const long long units = (long long)c.batch * c.Hkv * ((c.n_tokens * (long long)c.G + v.rows - 1) / v.rows);
  return v.max_tiles(c, units) <= 0x7FFFFFFFll;   // tiles are counted in 32 bits
}

size_t paged_mma_bytes(const PagedCache& c, int sm_count) {
  Variant v;
  if (!pick(c, &v)) return 0;
  return (size_t)2 * v.per_sm * sm_count * v.rows * (v.d + 2) * sizeof(float);
}

cudaError_t launch_paged_mma(void* state, const PagedCache& c, const RowsView& Q, void* out, float* lse, float* part, int sm_count,
                             const int (*clusters_of)[5], long long wait_limit, cudaStream_t st, int* launches) {
  Variant v;
  if (!pick(c, &v)) return cudaErrorInvalidValue;
  CUtensorMap tmK{}, tmV{};
  if (c.format == RESTKV_PAGES_BF16) {
    const cuuint64_t dims[2] = {(cuuint64_t)c.d, (cuuint64_t)c.n_pages * c.Hkv * c.page_rows};
    const cuuint64_t str[1] = {(cuuint64_t)c.d * 2};
    if (encode_tiles((TcState*)state, &tmK, c.K, 2, dims, str, kBlockRows) != CUDA_SUCCESS ||
        encode_tiles((TcState*)state, &tmV, c.V, 2, dims, str, kBlockRows) != CUDA_SUCCESS)
      return cudaErrorInvalidValue;
  }
  PagedMmaArgs a{};
  a.c = c; a.Q = Q; a.out = (__nv_bfloat16*)out; a.lse = lse; a.part = part; a.wait_limit = wait_limit;
  a.row_tiles = (c.n_tokens * c.G + v.rows - 1) / v.rows;
  const long long units = (long long)c.batch * c.Hkv * a.row_tiles;
  a.cluster = paged_mma_cluster(c, v, units, clusters_of[v.per_sm - 1]);
  *launches = 1;
  if (a.cluster) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned int)(units * a.cluster));
    cfg.blockDim = dim3((unsigned int)v.threads);
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
  int ctas = v.per_sm * sm_count;
  if (ctas > kMaxCtas) ctas = kMaxCtas;
  const cudaError_t e = launch_chained(v.kernel, dim3((unsigned int)ctas), v.threads, v.smem, st, tmK, tmV, a);
  if (e != cudaSuccess) return e;
  *launches = 2;
  return launch_chained(v.combine, dim3((unsigned int)units, (unsigned int)v.rows), 2 * v.d, 0, st, a, ctas, v.tile_rows);
}

}  // namespace restkv
