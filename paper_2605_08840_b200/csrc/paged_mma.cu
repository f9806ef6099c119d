// Attention of a few query tokens over the paged cache: bf16 in and out, pages of bf16 or of 4-bit codes, head_dim 64, 128 or 256.
//
// What bounds it: every row is read once and meets few query rows (tokens x query heads of a KV head, up to 16 per pass), so the step
// streams HBM; in 4 bits the instructions that turn codes into operands come close behind.  The design follows from that:
//   - warps that never wait for one another while they stream: each owns every kWarps-th tile of its CTA's run and a ring of tile
//     slots that its own lane 0 fills with bulk copies (4 bits: a block of 16 rows lies in one piece, codes and parameters) or TMA
//     boxes (bf16: 128-byte swizzle for ldmatrix);
//   - mma.sync m16n8k16: S = Q K^T with the query rows as the 16 rows and 8 cache rows as columns, O^T = V^T P^T with 16 dims as rows
//     and 8 query rows as columns.  The accumulator layout of S is the operand layout of P^T, so the weights never leave the
//     registers, and up to 8 query rows cost half of what P V with 16 padded rows does;
//   - 4-bit rows are laid out for the fragments: a lane's 4 bytes of K are 8 codes of the dims that its operand registers take, its 2
//     bytes of V 4 dims of one row.
//     A nibble is an operand as it stands: the 16 bits c << 4k are the f16 subnormal 2^(4k - 24) c for k = 0, 1, products with it are
//     exact in the fp32 accumulator, and a shift and four logic operations make 4 operand registers of 8 codes.  q is f16 scaled by a
//     power of two per query row (exact down to 2^-28 of the row's largest element).  s = step * (q . code) + offset * sum(q) per
//     group, o = sum f16(p step) code + sum p offset, all sums in fp32.
//     (bf16 16 + code: two operations per register, and the weights' rounding weighs twice as much unless 8 is taken off the codes:
//     60 us for 131072 rows.  e4m3 codes: m16n8k32 is carried out as conversions and f16 products here, 60 us, too.)
// Work is split in one of two ways:
//   - a cluster of CTAs per unit (sequence, KV head, up to 16 query rows), merged through distributed shared memory: one launch, for
//     short caches, where latency counts;
//   - the tiles of all units end to end, an equal share of them per CTA whatever the sequences' lengths, partial results in the
//     workspace and a second kernel that merges what several CTAs share.
#include <math.h>

#include <type_traits>

#include <cooperative_groups.h>
#include <cuda_fp16.h>

#include "paged.cuh"
#include "tc_common.cuh"

namespace restkv {

namespace {

namespace cg = cooperative_groups;

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
__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
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
__device__ __forceinline__ float lower(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float upper(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

struct PagedMmaArgs {
  PagedCache c;
  RowsView Q;
  __nv_bfloat16* out;
  float* lse;        // or null
  float* part;       // per CTA two of: o [rows, d], (m, l) [rows]; without clusters
  int row_tiles;     // units per KV head
  int cluster;       // CTAs per unit, 0: tiles of all units end to end
  long long wait_limit;
};

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
  static_assert(kRing >= kPartBytes + (kRows + kWarps - 1) / kWarps * kD * 4u, "the merge needs the ring's space");
  static constexpr size_t kSmem = (size_t)kWarps * kRing + 1024;
};

// Where a CTA's run of tiles begins: entry (a sequence, or with lengths per head a KV head of one), unit of the entry, tile of the unit.
struct Run {
  long long tiles;          // of all units
  long long first;          // tile at which `entry` begins
  int entry;
};

__device__ __forceinline__ int entry_tiles(const PagedCache& c, int e, int tile_rows) {
  const int n = c.per_head ? paged_length(c, e / c.Hkv, e % c.Hkv) : paged_length(c, e, 0);
  const int t = (n + tile_rows - 1) / tile_rows;
  return t > 0 ? t : 1;     // a unit without rows has its outputs written, too
}

// By a whole warp: the tiles of all units, and the entry that holds tile share(tiles).
template <typename F>
__device__ __forceinline__ Run find_run(const PagedCache& c, int row_tiles, int tile_rows, F share) {
  const int lane = threadIdx.x & 31;
  const int entries = c.per_head ? c.batch * c.Hkv : c.batch;
  const int units = c.per_head ? row_tiles : c.Hkv * row_tiles;
  Run r{0, 0, 0};
  long long mine = 0;
  for (int e = lane; e < entries; e += 32) mine += (long long)entry_tiles(c, e, tile_rows) * units;
  r.tiles = mine;
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) r.tiles += __shfl_xor_sync(0xffffffffu, r.tiles, off);
  const long long want = share(r.tiles);
  for (int base = 0; base < entries; base += 32) {
    const long long t = base + lane < entries ? (long long)entry_tiles(c, base + lane, tile_rows) * units : 0;
    long long upto = t;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const long long o = __shfl_up_sync(0xffffffffu, upto, off);
      if (lane >= off) upto += o;
    }
    const unsigned int past = __ballot_sync(0xffffffffu, r.first + upto > want);
    if (past) {
      const int at = __ffs((int)past) - 1;
      r.entry = base + at;
      r.first += __shfl_sync(0xffffffffu, upto - t, at);
      return r;
    }
    r.first += __shfl_sync(0xffffffffu, upto, 31);
  }
  r.entry = entries;
  return r;
}

template <int kD, int kGroups, int kNT>
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
  __shared__ float w_lo[kW][kRows][kG];        // 4 bits: sum of p offset per group
  __shared__ float c_ml[kRows][2];
  __shared__ int abort_flag;
  __shared__ long long run_s[2];
  __shared__ int run_entry;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, r = lane >> 2, q4 = lane & 3;
  const uint32_t smem_base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* rings = smem_raw + (smem_base - smem_u32(smem_raw));
  uint8_t* ring = rings + warp * C::kRing;
  const uint32_t ring_addr = smem_base + (uint32_t)warp * C::kRing;
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
  grid_dependency_wait();
  grid_dependency_launch();

  long long tile = 0, end = 0, first = 0;      // of the CTA's run, without clusters
  int entry = 0;
  if (!a.cluster) {
    if (warp == 0) {
      const Run run = find_run(c, a.row_tiles, C::kTileRows, [&](long long t) {
        return blockIdx.x < t ? t * blockIdx.x / (t < gridDim.x ? t : gridDim.x) : 0;
      });
      if (lane == 0) { run_s[0] = run.tiles; run_s[1] = run.first; run_entry = run.entry; }
    }
    __syncthreads();
    const long long ctas = run_s[0] < gridDim.x ? run_s[0] : gridDim.x;     // of them each has a tile
    if (blockIdx.x >= ctas) return;
    tile = run_s[0] * blockIdx.x / ctas;
    end = run_s[0] * (blockIdx.x + 1) / ctas;
    first = run_s[1];
    entry = run_entry;
  } else {
    __syncthreads();
  }

  int slot = 0;                                // of the warp's ring: the next tile's, and the parity it completes with
  uint32_t parity = 0;
  bool ok = true;
  for (int piece = 0;; ++piece) {
    // ---- the unit and the run of its tiles ----
    int unit, t0, t1, whole;                   // whole: no other CTA has tiles of the unit
    int cluster_rank = 0;
    if (a.cluster) {
      unit = (int)(blockIdx.x / (unsigned int)a.cluster);
      cluster_rank = (int)(blockIdx.x % (unsigned int)a.cluster);
      const int bh = unit / a.row_tiles;
      const int tiles = entry_tiles(c, c.per_head ? bh : bh / c.Hkv, C::kTileRows);
      t0 = (int)((long long)tiles * cluster_rank / a.cluster);
      t1 = (int)((long long)tiles * (cluster_rank + 1) / a.cluster);
      whole = 0;
    } else {
      const int units = c.per_head ? a.row_tiles : c.Hkv * a.row_tiles;
      int tiles = entry_tiles(c, entry, C::kTileRows);
      if (tile >= first + (long long)tiles * units) {      // the next entry
        first += (long long)tiles * units;
        ++entry;
        tiles = entry_tiles(c, entry, C::kTileRows);
      }
      const int k = (int)((tile - first) / tiles);
      const long long begin = first + (long long)k * tiles;
      unit = entry * units + k;
      t0 = (int)(tile - begin);
      t1 = (int)((end - begin < tiles) ? end - begin : tiles);
      whole = t0 == 0 && t1 == tiles;
    }
    const int bh = unit / a.row_tiles, rho0 = (unit - bh * a.row_tiles) * kRows, b = bh / c.Hkv, h = bh - b * c.Hkv;
    const int n = paged_length(c, b, h), count = paged_count(c, b);
    if (t0 == 0 && threadIdx.x == 0) check_length(c, b, h);
    const int blocks = (n + kBlockRows - 1) / kBlockRows;
    const int mine = t1 - t0 > warp ? (t1 - t0 - warp + kW - 1) / kW : 0;   // tiles t0 + warp + kW * i

    // ---- requests: the blocks' places are looked up 32 / kBlocks tiles at a time, one lane each ----
    int place = -1;
    unsigned int absent = 0;                   // bit slot * kBlocks + block: nothing was loaded there
    auto request = [&](int i, int s) {         // tile i into slot s, by the whole warp
      constexpr int kAhead = 32 / kBlocks;
      if (i % kAhead == 0) {
        const int t = t0 + warp + (i + lane / kBlocks) * kW;
        const int block = t * kBlocks + lane % kBlocks;
        place = -1;
        if (t < t1 && block < blocks) {
          place = paged_block_index(c, b, h, block);
          if (place < 0) atomicOr(c.dev_status, kDevBadIndex);
        }
      }
      int at[kBlocks];
      int there = 0;
#pragma unroll
      for (int k = 0; k < kBlocks; ++k) {
        at[k] = __shfl_sync(0xffffffffu, place, (i % kAhead) * kBlocks + k);
        there += at[k] >= 0;
        const unsigned int bit = 1u << (s * kBlocks + k);
        absent = at[k] >= 0 ? absent & ~bit : absent | bit;
      }
      if (lane == 0) {
        uint8_t* dst = ring + (uint32_t)s * C::kStageBytes;
        uint64_t* bar = &full[warp][s];
        mbar_arrive_expect_tx(bar, (uint32_t)there * 2 * C::kBlockBytes);
        if constexpr (kInt4) {
          // K's blocks, then V's; two that follow one another in a page come in one piece
          if (kBlocks == 2 && at[0] >= 0 && at[kBlocks - 1] == at[0] + 1) {
            bulk_load(dst, c.K + (long long)at[0] * C::kBlockBytes, 2 * C::kBlockBytes, bar);
            bulk_load(dst + 2 * C::kBlockBytes, c.V + (long long)at[0] * C::kBlockBytes, 2 * C::kBlockBytes, bar);
          } else {
#pragma unroll
            for (int k = 0; k < kBlocks; ++k) {
              if (at[k] < 0) continue;
              bulk_load(dst + k * C::kBlockBytes, c.K + (long long)at[k] * C::kBlockBytes, C::kBlockBytes, bar);
              bulk_load(dst + (kBlocks + k) * C::kBlockBytes, c.V + (long long)at[k] * C::kBlockBytes, C::kBlockBytes, bar);
            }
          }
        } else {
#pragma unroll
          for (int k = 0; k < kBlocks; ++k) {
            if (at[k] < 0) continue;
#pragma unroll
            for (int x = 0; x < kD / 64; ++x) {
              tma_load_2d(dst + k * C::kBlockBytes + x * 2048, &tmK, bar, x * 64, at[k] * kBlockRows);
              tma_load_2d(dst + (kBlocks + k) * C::kBlockBytes + x * 2048, &tmV, bar, x * 64, at[k] * kBlockRows);
            }
          }
        }
      }
      __syncwarp();
    };
#pragma unroll
    for (int i = 0; i < kStages; ++i)
      if (i < mine) request(i, slot + i < kStages ? slot + i : slot + i - kStages);

    // ---- Q as the A operand: query rows rho0 + r (and + 8), kD / 16 steps; what each row sees ----
    // 4 bits: in f16, scaled by a power of two per row (and 2^-4 where the codes come 16 times too large); sums of q per group in the
    // codes' and that scale, which the logits' factor takes out again.
    uint32_t qa[kD / 16][2 * kNT];
    float q_sum[kNT][kG], unscale[kNT];
    int sees[kNT];
    int sees_least = n;
#pragma unroll
    for (int t = 0; t < kNT; ++t) {
      const int rho = rho0 + r + 8 * t, i = rho / c.G, g = rho - i * c.G;
      const bool live = rho < R && i < count;
      sees[t] = live ? n - (count - 1 - i) : n;
      sees_least = min(sees_least, sees[t]);
      unscale[t] = 1.f;
      const __nv_bfloat16* q = reinterpret_cast<const __nv_bfloat16*>(a.Q.data) + b * a.Q.sb + (long long)(h * c.G + g) * a.Q.sh + i * a.Q.sn;
      if constexpr (kInt4) {
        uint4 u[kWords];                       // dims 32 m + 8 q4 .. + 7
        float top = 0.f;
#pragma unroll
        for (int m = 0; m < kWords; ++m) {
          u[m] = live ? *reinterpret_cast<const uint4*>(q + 32 * m + 8 * q4) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
          for (int x = 0; x < 4; ++x) top = fmaxf(top, fmaxf(fabsf(lower((&u[m].x)[x])), fabsf(upper((&u[m].x)[x]))));
        }
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
        // 2^e top in [2^14, 2^15), for top of 2^-86 .. 2^100; an infinite one makes the row's logits NaN
        int e = 141 - (int)(__float_as_uint(top) >> 23);
        e = e < -100 ? -100 : e > 100 ? 100 : e;
        const float scale = top < INFINITY ? __uint_as_float((uint32_t)(127 + e) << 23) : __uint_as_float(0x7FFFFFFFu);
        unscale[t] = __uint_as_float((uint32_t)(127 + 24 - e) << 23);
#pragma unroll
        for (int g2 = 0; g2 < kG; ++g2) q_sum[t][g2] = 0.f;
#pragma unroll
        for (int m = 0; m < kWords; ++m) {
          float v[8];
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            v[2 * x] = lower((&u[m].x)[x]) * scale;
            v[2 * x + 1] = upper((&u[m].x)[x]) * scale;
          }
          // the pairs (i, i + 4) that a word's codes come in
          qa[2 * m][t] = pack_f16x2(v[0], v[4]);
          qa[2 * m][kNT + t] = pack_f16x2(0x1p-4f * v[1], 0x1p-4f * v[5]);
          qa[2 * m + 1][t] = pack_f16x2(v[2], v[6]);
          qa[2 * m + 1][kNT + t] = pack_f16x2(0x1p-4f * v[3], 0x1p-4f * v[7]);
          q_sum[t][m / kPerGroup] += ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
        }
#pragma unroll
        for (int g2 = 0; g2 < kG; ++g2) {
          q_sum[t][g2] += __shfl_xor_sync(0xffffffffu, q_sum[t][g2], 1);
          q_sum[t][g2] += __shfl_xor_sync(0xffffffffu, q_sum[t][g2], 2);
          q_sum[t][g2] *= 0x1p-24f;
        }
      } else {
#pragma unroll
        for (int k = 0; k < kD / 16; ++k) {
          qa[k][t] = live ? *reinterpret_cast<const uint32_t*>(q + 16 * k + 2 * q4) : 0u;
          qa[k][kNT + t] = live ? *reinterpret_cast<const uint32_t*>(q + 16 * k + 8 + 2 * q4) : 0u;
        }
      }
    }
    sees_least = __reduce_min_sync(0xffffffffu, sees_least);

    const float cap_log2 = c.softcap * kLog2e;
    float to_log2[kNT];                        // what a row's sums are multiplied with: to log2 units, or to the cap's exponent
#pragma unroll
    for (int t = 0; t < kNT; ++t)
      to_log2[t] = (c.softcap > 0.f ? 2.f * kLog2e * c.scale / c.softcap : c.scale * kLog2e) * unscale[t];
    float ref[kNT], l[kNT];                    // weights are 2^(logit - ref); l: this lane's share of the row's sum
    float o[kD / 16][kNT][4];                  // dims of the 16-dim tile (r, r + 8), query rows 2 q4, 2 q4 + 1 (+ 8 per tile)
    float lo[kG][kNT];                         // 4 bits: this lane's share of sum p offset
#pragma unroll
    for (int t = 0; t < kNT; ++t) {
      ref[t] = -INFINITY;
      l[t] = 0.f;
#pragma unroll
      for (int k = 0; k < kD / 16; ++k)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[k][t][e] = 0.f;
#pragma unroll
      for (int g = 0; g < kG; ++g) lo[g][t] = 0.f;
    }

    // One tile; kEdge: some of its rows are not there, or not for every query row.
    auto take = [&](auto edge, uint32_t stage, int row0, unsigned int gone) {
      constexpr bool kEdge = decltype(edge)::value;
      // rows of the lane's four columns in a block: 4 bits q4 + 4 j, which is the order of the parameters; bf16 2 q4 + (j & 1) + 8 (j / 2)
      auto column = [&](int j) { return kInt4 ? q4 + 4 * j : 2 * q4 + (j & 1) + 8 * (j >> 1); };
      float sc[kBlocks][kNT][4];
#pragma unroll
      for (int k = 0; k < kBlocks; ++k) {
        const uint32_t kt = stage + k * C::kBlockBytes;
        if constexpr (kInt4) {
          uint32_t w[2][kWords];               // rows r / 2 + 4 (r % 2) (+ 8): columns r of the two tiles of 8 columns
#pragma unroll
          for (int half = 0; half < 2; ++half)
            lds_words<kWords>(kt + (uint32_t)(8 * half + (r >> 1) + 4 * (r & 1)) * (kD / 2) + q4 * (kD / 8), w[half]);
#pragma unroll
          for (int g = 0; g < kG; ++g) {
            float acc[2][4];                   // rows r, r + 8; columns 2 q4, 2 q4 + 1
#pragma unroll
            for (int half = 0; half < 2; ++half)
#pragma unroll
              for (int x = g * kPerGroup; x < (g + 1) * kPerGroup; ++x) {
                const uint32_t a0[4] = {qa[2 * x][0], kNT == 2 ? qa[2 * x][1] : 0u, qa[2 * x][kNT], kNT == 2 ? qa[2 * x][kNT + kNT - 1] : 0u};
                const uint32_t a1[4] = {qa[2 * x + 1][0], kNT == 2 ? qa[2 * x + 1][1] : 0u, qa[2 * x + 1][kNT],
                                        kNT == 2 ? qa[2 * x + 1][kNT + kNT - 1] : 0u};
                if (x == g * kPerGroup) mma16816_f16_start(acc[half], a0, code_pair<0>(w[half][x]), code_pair<1>(w[half][x]));
                else mma16816_f16(acc[half], a0, code_pair<0>(w[half][x]), code_pair<1>(w[half][x]));
                mma16816_f16(acc[half], a1, code_pair<2>(w[half][x]), code_pair<3>(w[half][x]));
              }
            const uint4 u = lds128(kt + 8 * kD + 64 * g + 16 * q4);
            const float step[4] = {lower(u.x), upper(u.x), lower(u.y), upper(u.y)}, off[4] = {lower(u.z), upper(u.z), lower(u.w), upper(u.w)};
#pragma unroll
            for (int t = 0; t < kNT; ++t)
#pragma unroll
              for (int j = 0; j < 4; ++j)
                sc[k][t][j] = fmaf(step[j], acc[j >> 1][2 * t + (j & 1)], g == 0 ? off[j] * q_sum[t][g] : fmaf(off[j], q_sum[t][g], sc[k][t][j]));
          }
        } else {
          float acc[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
          const int mat = lane >> 3, mr = lane & 7;
#pragma unroll
          for (int x = 0; x < kD / 16; ++x) {
            uint32_t w[4];
            ldsm4(kt + (uint32_t)(x >> 2) * 2048u + (uint32_t)((mat >> 1) * 8 + mr) * 128u + (((uint32_t)((x & 3) * 2 + (mat & 1)) ^ (uint32_t)mr) << 4), w);
            const uint32_t a0[4] = {qa[x][0], kNT == 2 ? qa[x][1] : 0u, qa[x][kNT], kNT == 2 ? qa[x][kNT + kNT - 1] : 0u};
            mma16816(acc[0], a0, w[0], w[1]);
            mma16816(acc[1], a0, w[2], w[3]);
          }
#pragma unroll
          for (int t = 0; t < kNT; ++t)
#pragma unroll
            for (int j = 0; j < 4; ++j) sc[k][t][j] = acc[j >> 1][2 * t + (j & 1)];
        }
      }
      // logits in log2 units; columns that a row does not see weigh nothing
#pragma unroll
      for (int k = 0; k < kBlocks; ++k)
#pragma unroll
        for (int t = 0; t < kNT; ++t)
#pragma unroll
          for (int j = 0; j < 4; ++j) sc[k][t][j] *= to_log2[t];
      if (cap_log2 > 0.f) {
        // cap * tanh(x / cap) with tanh(y) = 1 - 2 / (1 + e^2y): 2^-22 of the cap
#pragma unroll
        for (int k = 0; k < kBlocks; ++k)
#pragma unroll
          for (int t = 0; t < kNT; ++t)
#pragma unroll
            for (int j = 0; j < 4; ++j) sc[k][t][j] = fmaf(-2.f * cap_log2, rcp_approx(1.f + ex2_approx(sc[k][t][j])), cap_log2);
      }
      if constexpr (kEdge) {
#pragma unroll
        for (int k = 0; k < kBlocks; ++k)
#pragma unroll
          for (int t = 0; t < kNT; ++t)
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (row0 + k * kBlockRows + column(j) >= sees[t] || (gone >> k & 1u)) sc[k][t][j] = -INFINITY;
      }
      // bits of the rows of V that are there
      uint32_t keep01[kBlocks], keep23[kBlocks];
#pragma unroll
      for (int k = 0; k < kBlocks; ++k) {
        keep01[k] = keep23[k] = 0xFFFFFFFFu;
        if constexpr (kEdge) {
          // rows past the cache hold anything: their bits are cleared, so that a weight of 0 finds a number there
          const int left = (gone >> k & 1u) ? 0 : n - (row0 + k * kBlockRows);
          keep01[k] = (column(0) < left ? 0xFFFFu : 0u) | (column(1) < left ? 0xFFFF0000u : 0u);
          keep23[k] = (column(2) < left ? 0xFFFFu : 0u) | (column(3) < left ? 0xFFFF0000u : 0u);
        }
      }
      // 4 bits: p step is to fit f16 whatever the steps are, so that the reference grows with the largest of them, too
      uint2 v_step[kBlocks][kG];
      float most = 0.f;
      if constexpr (kInt4) {
        uint32_t top = 0x2B802B80u;            // 2^-40 at least: weights stay well within fp32
#pragma unroll
        for (int k = 0; k < kBlocks; ++k)
#pragma unroll
          for (int g = 0; g < kG; ++g) {
            v_step[k][g] = lds64(stage + (kBlocks + k) * C::kBlockBytes + 8 * kD + 64 * g + 16 * q4);
            v_step[k][g].x &= keep01[k];
            v_step[k][g].y &= keep23[k];
            top = __vmaxu2(top, __vmaxu2(v_step[k][g].x, v_step[k][g].y));   // steps are not negative: ordered as integers
          }
        most = lg2_approx(__uint_as_float(max(top & 0xFFFF0000u, top << 16)));
      }
      float f[kNT];
      bool grown = false;
#pragma unroll
      for (int t = 0; t < kNT; ++t) {
        float mx = -INFINITY;
#pragma unroll
        for (int k = 0; k < kBlocks; ++k) mx = fmaxf(mx, fmaxf(fmaxf(sc[k][t][0], sc[k][t][1]), fmaxf(sc[k][t][2], sc[k][t][3])));
        mx += most;
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
        f[t] = 1.f;
        if (mx > ref[t] + kSlack) {            // o is rescaled only when the weights would grow past 2^kSlack
          f[t] = ex2_approx(ref[t] - (mx - kStart));   // ref = -inf gives 0
          ref[t] = mx - kStart;
          l[t] *= f[t];
          grown = true;
        }
        const float m_use = ref[t] == -INFINITY ? 0.f : ref[t];   // only logits of -inf so far: they weigh nothing
#pragma unroll
        for (int k = 0; k < kBlocks; ++k) {
#pragma unroll
          for (int j = 0; j < 4; ++j) sc[k][t][j] = ex2_approx(sc[k][t][j] - m_use);
          l[t] += (sc[k][t][0] + sc[k][t][1]) + (sc[k][t][2] + sc[k][t][3]);
        }
      }
      if (__any_sync(0xffffffffu, grown)) {
#pragma unroll
        for (int t = 0; t < kNT; ++t) {
          // the factors of the rows that o's columns stand for
          const float f0 = __shfl_sync(0xffffffffu, f[t], 8 * q4), f1 = __shfl_sync(0xffffffffu, f[t], 8 * q4 + 4);
#pragma unroll
          for (int k = 0; k < kD / 16; ++k) {
            o[k][t][0] *= f0; o[k][t][1] *= f1;
            o[k][t][2] *= f0; o[k][t][3] *= f1;
          }
          if (kInt4) {
#pragma unroll
            for (int g = 0; g < kG; ++g) lo[g][t] *= f[t];
          }
        }
      }
#pragma unroll
      for (int k = 0; k < kBlocks; ++k) {
        const uint32_t vt = stage + (kBlocks + k) * C::kBlockBytes;
        if constexpr (kInt4) {
          uint32_t w[4][(kWords + 1) / 2];     // the units of rows q4, q4 + 4, q4 + 8, q4 + 12
#pragma unroll
          for (int j = 0; j < 4; ++j) lds_words<kWords / 2>(vt + (uint32_t)(q4 + 4 * j) * (kD / 2) + r * (kD / 16), w[j]);
          uint32_t pb[kNT][2];
#pragma unroll
          for (int x = 0; x < kWords; ++x) {
            if (x % kPerGroup == 0) {
              const int g = x / kPerGroup;
              uint2 u = lds64(vt + 8 * kD + 64 * g + 16 * q4 + 8);
              if constexpr (kEdge) { u.x &= keep01[k]; u.y &= keep23[k]; }
              const float s0 = lower(v_step[k][g].x), s1 = upper(v_step[k][g].x), s2 = lower(v_step[k][g].y), s3 = upper(v_step[k][g].y);
#pragma unroll
              for (int t = 0; t < kNT; ++t) {
                const float* p = sc[k][t];
                lo[g][t] = fmaf(p[0], lower(u.x), fmaf(p[1], upper(u.x), fmaf(p[2], lower(u.y), fmaf(p[3], upper(u.y), lo[g][t]))));
                pb[t][0] = pack_f16x2(p[0] * s0, p[1] * s1);
                pb[t][1] = pack_f16x2(p[2] * s2, p[3] * s3);
              }
            }
            const uint32_t y0 = __byte_perm(w[0][x >> 1], w[1][x >> 1], x & 1 ? 0x7632 : 0x5410);
            const uint32_t y1 = __byte_perm(w[2][x >> 1], w[3][x >> 1], x & 1 ? 0x7632 : 0x5410);
            const uint32_t va[4] = {code_pair<0>(y0), code_pair<1>(y0), code_pair<0>(y1), code_pair<1>(y1)};
            const uint32_t vb[4] = {code_pair<2>(y0), code_pair<3>(y0), code_pair<2>(y1), code_pair<3>(y1)};
#pragma unroll
            for (int t = 0; t < kNT; ++t) {
              mma16816_f16(o[2 * x][t], va, pb[t][0], pb[t][1]);
              mma16816_f16(o[2 * x + 1][t], vb, pb[t][0], pb[t][1]);
            }
          }
        } else {
          uint32_t pb[kNT][2];
#pragma unroll
          for (int t = 0; t < kNT; ++t) {
            pb[t][0] = pack_bf16x2(sc[k][t][0], sc[k][t][1]);
            pb[t][1] = pack_bf16x2(sc[k][t][2], sc[k][t][3]);
          }
          const int mat = lane >> 3, mr = lane & 7;
#pragma unroll
          for (int x = 0; x < kD / 16; ++x) {
            uint32_t va[4];
            ldsm4_t(vt + (uint32_t)(x >> 2) * 2048u + (uint32_t)((mat >> 1) * 8 + mr) * 128u + (((uint32_t)((x & 3) * 2 + (mat & 1)) ^ (uint32_t)mr) << 4), va);
            if constexpr (kEdge) { va[0] &= keep01[k]; va[1] &= keep01[k]; va[2] &= keep23[k]; va[3] &= keep23[k]; }
#pragma unroll
            for (int t = 0; t < kNT; ++t) mma16816(o[x][t], va, pb[t][0], pb[t][1]);
          }
        }
      }
    };

    for (int i = 0; i < mine; ++i) {
      ok = __all_sync(0xffffffffu, mbar_wait(&full[warp][slot], parity, &abort_flag, c.dev_status, kDevTimeout, a.wait_limit));
      if (!ok) {
        if (lane == 0)   // nothing may still be on its way into shared memory when the CTA returns
          for (int j = 0; j < kStages && i + j < mine; ++j) {
            const int s = slot + j < kStages ? slot + j : slot + j - kStages;
            wait_issued(&full[warp][s], s < slot ? parity ^ 1u : parity);
          }
        break;
      }
      const uint32_t stage = ring_addr + (uint32_t)slot * C::kStageBytes;
      const int row0 = (t0 + warp + i * kW) * C::kTileRows;
      const unsigned int gone = absent >> (slot * kBlocks) & ((1u << kBlocks) - 1u);
      if (row0 + C::kTileRows > sees_least || gone != 0) take(std::true_type{}, stage, row0, gone);
      else take(std::false_type{}, stage, row0, 0u);
      __syncwarp();   // every lane has read the slot
      if (i + kStages < mine) request(i + kStages, slot);
      if (++slot == kStages) { slot = 0; parity ^= 1u; }
    }

    // ---- merge, in a fixed order: the warps of the CTA through their (idle) rings ----
    __syncwarp();
    float* w_o = reinterpret_cast<float*>(ring);   // [rows][kD]
#pragma unroll
    for (int t = 0; t < kNT; ++t) {
      l[t] += __shfl_xor_sync(0xffffffffu, l[t], 1);
      l[t] += __shfl_xor_sync(0xffffffffu, l[t], 2);
      if (q4 == 0) { w_ml[warp][r + 8 * t][0] = ref[t]; w_ml[warp][r + 8 * t][1] = l[t]; }
      if (kInt4) {
#pragma unroll
        for (int g = 0; g < kG; ++g) {
          lo[g][t] += __shfl_xor_sync(0xffffffffu, lo[g][t], 1);
          lo[g][t] += __shfl_xor_sync(0xffffffffu, lo[g][t], 2);
          if (q4 == 0) w_lo[warp][r + 8 * t][g] = lo[g][t];
        }
      }
      if (mine > 0) {
        float* row = w_o + (2 * q4 + 8 * t) * kD;
        if constexpr (kInt4) {
#pragma unroll
          for (int x = 0; x < kWords; ++x) {   // dims 32 x + 4 r + (0..3)
            const float *e = o[2 * x][t], *f = o[2 * x + 1][t];
            *reinterpret_cast<float4*>(row + 32 * x + 4 * r) = make_float4(e[0] * 0x1p24f, e[2] * 0x1p20f, f[0] * 0x1p24f, f[2] * 0x1p20f);
            *reinterpret_cast<float4*>(row + kD + 32 * x + 4 * r) = make_float4(e[1] * 0x1p24f, e[3] * 0x1p20f, f[1] * 0x1p24f, f[3] * 0x1p20f);
          }
        } else {
#pragma unroll
          for (int x = 0; x < kD / 16; ++x) {
            row[16 * x + r] = o[x][t][0];
            row[kD + 16 * x + r] = o[x][t][1];
            row[16 * x + 8 + r] = o[x][t][2];
            row[kD + 16 * x + 8 + r] = o[x][t][3];
          }
        }
      }
    }
    __syncthreads();
    const int rows = R - rho0 < kRows ? R - rho0 : kRows;
    // a row's result: written where the unit is this CTA's (or this cluster's) alone
    auto finish = [&](int row, int k, float acc, float mm, float ll) {
      const int rho = rho0 + row, i = rho / c.G, g = rho - i * c.G;
      const bool some = ll > 0.f && i < count;
      const long long at = ((long long)b * c.Hq + h * c.G + g) * c.n_tokens + i;
      a.out[at * kD + k] = __float2bfloat16(some ? acc / ll : 0.f);
      if (k == 0 && a.lse) a.lse[at] = some ? fmaf(mm, 0.6931471805599453f, logf(ll)) : -INFINITY;
    };
    auto c_o = [&](int row) { return reinterpret_cast<float*>(rings + (row % kW) * C::kRing + C::kPartBytes) + (row / kW) * kD; };
    for (int e = threadIdx.x; e < rows * kD; e += kW * 32) {
      const int row = e / kD, k = e % kD;
      float mm = -INFINITY;
#pragma unroll
      for (int w = 0; w < kW; ++w) mm = fmaxf(mm, w_ml[w][row][0]);
      float acc = 0.f, ll = 0.f;
#pragma unroll
      for (int w = 0; w < kW; ++w) {
        const float mw = w_ml[w][row][0];
        if (mw == -INFINITY) continue;         // a warp without tiles, or whose tiles this row does not see
        const float f = ex2_approx(mw - mm);
        float v = reinterpret_cast<const float*>(rings + w * C::kRing)[row * kD + k];
        if (kInt4) v += w_lo[w][row][k / (kD / kG)];
        acc = fmaf(v, f, acc);
        ll = fmaf(w_ml[w][row][1], f, ll);
      }
      if (a.cluster) {
        c_o(row)[k] = acc;
        if (k == 0) { c_ml[row][0] = mm; c_ml[row][1] = ll; }
      } else if (whole) {
        finish(row, k, acc, mm, ll);
      } else {
        float* p = a.part + (long long)(2 * blockIdx.x + (piece > 0)) * kRows * (kD + 2);
        p[row * kD + k] = acc;
        if (k == 0) { p[kRows * kD + 2 * row] = mm; p[kRows * kD + 2 * row + 1] = ll; }
      }
    }
    if (a.cluster) {
      cg::cluster_group cluster = cg::this_cluster();
      cluster.sync();
      for (int e = cluster_rank * kW * 32 + (int)threadIdx.x; e < rows * kD; e += a.cluster * kW * 32) {
        const int row = e / kD, k = e % kD;
        float mm = -INFINITY, acc = 0.f, ll = 0.f;
        float mr[16], lr[16], vr[16];
#pragma unroll
        for (int x = 0; x < 16; ++x) {
          mr[x] = -INFINITY;
          if (x < a.cluster) {
            const float* p = cluster.map_shared_rank(&c_ml[row][0], x);
            mr[x] = p[0];
            lr[x] = p[1];
            vr[x] = *cluster.map_shared_rank(c_o(row) + k, x);
            mm = fmaxf(mm, mr[x]);
          }
        }
#pragma unroll
        for (int x = 0; x < 16; ++x) {
          if (mr[x] == -INFINITY) continue;
          const float f = ex2_approx(mr[x] - mm);
          acc = fmaf(vr[x], f, acc);
          ll = fmaf(lr[x], f, ll);
        }
        finish(row, k, acc, mm, ll);
      }
      cluster.sync();   // shared memory stays alive until every peer has read it
      return;
    }
    tile += t1 - t0;
    // all of the CTA's warps go on to the next piece or none
    if (__syncthreads_or(!ok) || tile >= end) return;
    fence_proxy_async_smem();   // the rings were written by ordinary stores; bulk copies come next
  }
}

// grid (units, rows), block 2 kD: merges what several CTAs left of a unit, 8 pieces at a time (kD / 4 threads each).
constexpr int kMaxCtas = 512;

template <int kD, int kRows>
__global__ void __launch_bounds__(2 * kD) paged_mma_combine_kernel(const __grid_constant__ PagedMmaArgs a, int ctas, int tile_rows) {
  grid_dependency_wait();
  __shared__ long long run_s[2];
  const PagedCache& c = a.c;
  const int unit = blockIdx.x, row = blockIdx.y, bh = unit / a.row_tiles, rho = (unit - bh * a.row_tiles) * kRows + row;
  if (rho >= c.n_tokens * c.G) return;
  const int units = c.per_head ? a.row_tiles : c.Hkv * a.row_tiles, entry = unit / units;
  const int b = bh / c.Hkv, h = bh - b * c.Hkv, i = rho / c.G, g = rho - i * c.G;
  if (threadIdx.x < 32) {
    // where the unit's entry begins, by the same sums as in the kernel before
    long long before = 0, all = 0;
    const int entries = c.per_head ? c.batch * c.Hkv : c.batch;
    for (int e = threadIdx.x; e < entries; e += 32) {
      const long long t = (long long)entry_tiles(c, e, tile_rows) * units;
      all += t;
      if (e < entry) before += t;
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
      all += __shfl_xor_sync(0xffffffffu, all, off);
      before += __shfl_xor_sync(0xffffffffu, before, off);
    }
    if (threadIdx.x == 0) { run_s[0] = all; run_s[1] = before; }
  }
  __syncthreads();
  const long long all = run_s[0];
  const int tiles = entry_tiles(c, entry, tile_rows);
  const long long u0 = run_s[1] + (long long)(unit - entry * units) * tiles, u1 = u0 + tiles;
  if (ctas > all) ctas = (int)all;
  // the CTA whose share [all * x / ctas, all * (x + 1) / ctas) holds tile t
  auto holder = [&](long long t) { return (int)(((t + 1) * ctas - 1) / all); };
  const int x0 = holder(u0), x1 = holder(u1 - 1);
  if (x0 == x1) return;                        // it was one CTA's: written
  // a CTA's first piece lies in its first slot, its last in the second; x0's is a later one where the unit begins inside its share
  constexpr long long kSlot = kRows * (kD + 2);
  const bool later = all * x0 / ctas < u0;
  const int pieces = x1 - x0 + 1;
  auto piece = [&](int x) { return a.part + (2ll * (x0 + x) + (x == 0 && later)) * kSlot; };
  __shared__ float factor[kMaxCtas];
  __shared__ float of_warp[2][2 * kD / 32];
  __shared__ float4 acc_s[8][kD / 4];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  float mm = -INFINITY;
  for (int x = threadIdx.x; x < pieces; x += 2 * kD) mm = fmaxf(mm, piece(x)[kRows * kD + 2 * row]);
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) mm = fmaxf(mm, __shfl_xor_sync(0xffffffffu, mm, off));
  if (lane == 0) of_warp[0][warp] = mm;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 2 * kD / 32; ++w) mm = fmaxf(mm, of_warp[0][w]);
  float ll = 0.f;
  for (int x = threadIdx.x; x < pieces; x += 2 * kD) {
    const float* ml = piece(x) + kRows * kD + 2 * row;
    const float f = ml[0] == -INFINITY ? 0.f : ex2_approx(ml[0] - mm);
    factor[x] = f;
    ll = fmaf(ml[1], f, ll);
  }
#pragma unroll
  for (int off = 16; off > 0; off >>= 1) ll += __shfl_xor_sync(0xffffffffu, ll, off);
  if (lane == 0) of_warp[1][warp] = ll;
  __syncthreads();
  ll = 0.f;
#pragma unroll
  for (int w = 0; w < 2 * kD / 32; ++w) ll += of_warp[1][w];
  const int sub = threadIdx.x / (kD / 4), v = threadIdx.x % (kD / 4);
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int x = sub; x < pieces; x += 8) {
    const float4 o = reinterpret_cast<const float4*>(piece(x) + row * kD)[v];
    const float f = factor[x];
    acc.x = fmaf(o.x, f, acc.x); acc.y = fmaf(o.y, f, acc.y); acc.z = fmaf(o.z, f, acc.z); acc.w = fmaf(o.w, f, acc.w);
  }
  acc_s[sub][v] = acc;
  __syncthreads();
  if (threadIdx.x >= kD) return;
  float sum = 0.f;
#pragma unroll
  for (int x = 0; x < 8; ++x) sum += reinterpret_cast<const float*>(acc_s[x])[threadIdx.x];
  const bool some = ll > 0.f && i < paged_count(c, b);
  const long long at = ((long long)b * c.Hq + h * c.G + g) * c.n_tokens + i;
  a.out[at * kD + threadIdx.x] = __float2bfloat16(some ? sum / ll : 0.f);
  if (threadIdx.x == 0 && a.lse) a.lse[at] = some ? fmaf(mm, 0.6931471805599453f, logf(ll)) : -INFINITY;
}

// ---- host: one set of functions per instantiation ----
struct Variant {
  void (*kernel)(CUtensorMap, CUtensorMap, PagedMmaArgs);
  void (*combine)(PagedMmaArgs, int, int);
  int d, threads, per_sm, rows, tile_rows;
  size_t smem;
};

template <int kD, int kGroups, int kNT> Variant variant() {
  using C = Config<kD, kGroups, kNT>;
  return Variant{paged_mma_kernel<kD, kGroups, kNT>, paged_mma_combine_kernel<kD, C::kRows>, kD, C::kWarps * 32, C::kPerSm, C::kRows,
                 C::kTileRows, C::kSmem};
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

}  // namespace

cudaError_t paged_mma_init() {
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
        if (e == cudaSuccess) e = cudaFuncSetAttribute(v.kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        if (e != cudaSuccess) return e;
      }
  return cudaSuccess;
}

bool paged_mma_supported(const PagedCache& c) {
  Variant v;
  return pick(c, &v);
}

size_t paged_mma_bytes(const PagedCache& c, int sm_count) {
  Variant v;
  if (!pick(c, &v)) return 0;
  return (size_t)2 * v.per_sm * sm_count * v.rows * (v.d + 2) * sizeof(float);
}

cudaError_t launch_paged_mma(void* state, const PagedCache& c, const RowsView& Q, void* out, float* lse, float* part, int sm_count,
                             long long wait_limit, cudaStream_t st, int* launches) {
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
  a.cluster = 0;
  const int units = c.batch * c.Hkv * a.row_tiles;
  const int ctas = v.per_sm * sm_count < kMaxCtas ? v.per_sm * sm_count : kMaxCtas;
  cudaError_t e = launch_chained(v.kernel, dim3((unsigned int)ctas), v.threads, v.smem, st, tmK, tmV, a);
  if (e != cudaSuccess) return e;
  *launches = 2;
  return launch_chained(v.combine, dim3((unsigned int)units, (unsigned int)v.rows), 2 * v.d, 0, st, a, ctas, v.tile_rows);
}

}  // namespace restkv
