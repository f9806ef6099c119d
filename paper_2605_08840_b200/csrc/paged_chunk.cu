// Attention of many query tokens over the paged cache (a chunk of prompt): bf16 in and out, pages of bf16 or of 4-bit codes, head_dim 64
// or 128, on tcgen05.
//
// What bounds it: 4 * 128 * 128 * head_dim operations per 128 query rows and 128 cache rows are 1024 cycles of the tensor pipe at head_dim
// 128, and the exponentials as many of the special-function unit; between the two the softmax's chain of load, maximum, exponential, sum,
// store, about 1650 cycles per half tile of 64 columns (2500 with a cap), which nothing but another warp's work hides.  So
//   - a CTA per SM takes 256 query rows (tokens x query heads of a KV head) in two tiles of 128, each with a warpgroup of its own, a
//     thread per row; a tile of K and V serves both;
//   - a tile of logits is two halves of 64 columns, in turn: while a row's thread is at one, the other's weights meet V and its next
//     logits are made, so that a softmax warp always finds a half ready (whole tiles in turn: 863 us for 815 below, with a cap 1294 for 1095);
//   - one pass over a half: 64 logits in registers, their maximum against the running reference, the weights.  The reference is moved (sums
//     and O scaled by a power of two) only where weights would pass 2^13 (a first pass for the maximum: 975 us for 864);
//   - S (fp32) and O of both tiles fill the tensor memory's 512 columns at head_dim 128; P (16 bits) takes S's place and is the A operand
//     of P V there;
//   - seven warps fetch K and V, half a row per thread: bf16 by cp.async; codes become f16 operands with one fused operation per pair, the
//     nibble as it stands being the f16 subnormal 2^-24 code (2^-20 for the upper one of a byte).
//     K: step * (code - 8), times 2^(a - 24) for a tile's exponent a that just lets its largest step fit f16: at most 11 bits, exact. The
//     rest, (offset + 8 step) * sum(q) per group, is three more products of f16 parts (22 bits together), another 16 dims for all groups.
//     V: offset + step * code, rounded once to f16; its tiles' exponents go into the weights'.
//     (K rounded like V: 10% less of the tensor pipe, but logits lose 2^-12 of their terms.  In both, steps below 2^-8 of the largest of
//     their 128 rows lose bits.)
//   - weights are rounded to f16 (over 4 bits) or bf16 before they meet V, as an output of bf16 is in the end; their sums are fp32 sums of
//     the weights before that;
//   - dims within K's operand chunks are in the order in which they come out of a word, and Q's in the same; V's order is undone where O
//     is written.
//   - a capped logit's tanh is an odd polynomial on the FMA pipe while |s / cap| <= 0.6 for all rows and columns that a warp has in hand;
//     else the exponential form with two trips to the special-function unit, under large caps that or the polynomial one by one.
//     (A part of the exponentials by a polynomial, too: an eighth of them 825 us for 811, a quarter 853; exponentials by turns with the other
//     tile's: 678 us for 667, with a cap 1031 for 874; weights made beside the maximum and made again where it has moved: 707 for 667, with a
//     cap 828 for 879, but bf16 804 for 789, groups of 32 1104 for 1068.  The chain bounds it, not the unit.)
// The tiles that a unit's last query row sees, of all units end to end, are dealt out evenly; what several CTAs share is merged by a second
// kernel.  Measured, 2048 tokens of 32 heads of 128 (8 KV heads) over 18432 rows: bf16 671 us (870 TFLOP/s, tensor pipe 43% busy), 4 bits in
// groups of 128 667 us, of 32 804 us (the conversion of codes, a step and an offset per row and group, bounds that one); with a cap of 30 786,
// 839 and 1075 us, with one of 5, which the logits reach, 1148 and 1250.  2048 tokens and nothing before them 122 us; 48 tokens over 17000
// rows 53 us.  What the last merge rounds is little beside the rest; the tensor pipe's own fp32 sums cut off what is below their last place,
// which for values of one sign adds up to 6e-4 of them over 131072 rows and 1.2e-3 over 524288 (values around 0: nothing).
#include <math.h>

#include <cuda_fp16.h>

#include "paged_deal.cuh"

namespace restkv {

namespace {

constexpr int kChRows = 256;                 // query rows of a unit
constexpr int kChTile = 128;                 // cache rows of a tile
constexpr int kSoftmaxWarps = 8, kFetchWarps = 7;   // and one for the products: four warps per scheduler, 128 registers
constexpr int kChThreads = (kSoftmaxWarps + kFetchWarps + 1) * 32;
constexpr int kFetch = kFetchWarps * 32;
constexpr int kInfo = 4;                     // tiles whose factors are kept: the fetching warps are two ahead of the softmax at most
// Tiles that a CTA could go through while it ends one unit and begins another.  (2048 tokens alone: none 181 us, 2 147, 4 144, 8 136; 300
// tokens over 8700 rows: 116, 116, 115, 121.)
constexpr int kChSnap = 4;
// log2 of the largest weight that a rescaling leaves, and of what it may grow to before the next one
constexpr float kChStart = 5.f, kChSlack = 13.f;

// Up to this cap small logits may go by tanh_far, too: 2^-22 of the cap is 2^-16, a thirty-second of what rounds a weight here.  (One by one,
// logits on both sides of 0.6 of the cap: 18432 rows in groups of 128 1504 us for 1207, bf16 1387 for 1144.)
constexpr float kTanhFarAlone = 64.f;

struct ChunkBarriers {
  uint64_t q_full[2], s_full[2][2], p_full[2][2], pv_done[2][2], k_full[2], k_empty[2], v_full[2], v_empty[2], drained;
};

// Row `row`, 16-byte chunk `chunk` of a 16-bit operand tile of 128 rows: boxes of [128 rows x 64 elements], 128-byte swizzle.
__device__ __forceinline__ uint32_t operand_at(uint32_t tile, int row, int chunk) {
  return tile + (uint32_t)(chunk >> 3) * 16384u + (uint32_t)row * 128u + (uint32_t)(((chunk & 7) ^ (row & 7)) << 4);
}
__device__ __forceinline__ void sts128(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
__device__ __forceinline__ uint32_t hfma2(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t d;
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(c));
  return d;
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(127 + (e < -126 ? -126 : e > 127 ? 127 : e)) << 23); }
__device__ __forceinline__ void fetch_sync() { asm volatile("bar.sync 1, %0;" ::"n"(kFetch) : "memory"); }

// 8 codes of a word as operands: s * 2^-24 code + l, where s16 = s / 16, for the codes in the lower and in the upper half of the word.
__device__ __forceinline__ void operands_of(uint32_t w, uint32_t s, uint32_t s16, uint32_t l, uint32_t to) {
  const uint32_t w8 = w >> 8;
  sts128(to, hfma2(s, w & 0x000F000Fu, l), hfma2(s16, w & 0x00F000F0u, l), hfma2(s, w8 & 0x000F000Fu, l), hfma2(s16, w8 & 0x00F000F0u, l));
}

// Row `row` of an operand 16 elements deep, without swizzle: 8 rows of 16 bytes together, both halves of a row 128 bytes apart.
constexpr uint32_t kThinBytes = 128 * 32;
__device__ __forceinline__ uint32_t thin_at(uint32_t tile, int row) { return tile + (uint32_t)(row >> 3) * 256u + (uint32_t)(row & 7) * 16u; }
// x as the sum of two f16: in the lower and in the upper half.
__device__ __forceinline__ uint32_t split_f16(float x) {
  const __half hi = __float2half_rn(x);
  return pack_f16x2(__half2float(hi), x - __half2float(hi));
}

// `columns` fp32 columns of the thread's row of tensor memory times f.  By whole warps.
__device__ __noinline__ void rescale(uint32_t at, int columns, float f) {
  for (int x = 0; x < columns; x += 16) {
    float v[16];
    tmem_ld16(at + x, v);
    tmem_wait_ld();
    uint32_t w[16];
#pragma unroll
    for (int y = 0; y < 16; ++y) w[y] = __float_as_uint(v[y] * f);
    tmem_st16(at + x, w);
  }
  tmem_wait_st();
}

// Tiles that the last query row of a unit sees: those past them are nobody's business.
__device__ __forceinline__ int unit_tiles(const PagedCache& c, int row_tiles, int unit) {
  const int bh = unit / row_tiles, rho0 = (unit - bh * row_tiles) * kChRows, b = bh / c.Hkv, count = paged_count(c, b);
  if (rho0 >= count * c.G) return 0;
  const int i_last = (min(rho0 + kChRows, count * c.G) - 1) / c.G;
  const int seen = paged_length(c, b, bh - b * c.Hkv) - (count - 1 - i_last);
  return seen > 0 ? (seen + kChTile - 1) / kChTile : 0;
}

template <int kD, int kGroups> struct ChunkConfig {
  static constexpr bool kInt4 = kGroups > 0;
  static constexpr uint32_t kTileBytesD = 128u * kD * 2u;
  static constexpr size_t kSmem = 6 * (size_t)kTileBytesD + (kInt4 ? 4 * kThinBytes : 0) + 1024;   // two tiles of Q, two of K, two of V
};

// A kernel of its own for capped logits: with the cap in a branch rows in groups of 32 take 905 us for 803 (with a cap 1114 for 1071), others
// 0.5% more (with a cap bf16 817 for 790, groups of 128 863 for 875).
template <int kD, int kGroups, bool kCap>
__global__ void __launch_bounds__(kChThreads, 1) paged_chunk_kernel(const __grid_constant__ PagedMmaArgs a) {
  using C = ChunkConfig<kD, kGroups>;
  constexpr bool kInt4 = C::kInt4;
  constexpr int kWords = kD / 32, kG = kInt4 ? kGroups : 1, kPerGroup = kWords / kG;
  const PagedCache& c = a.c;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) ChunkBarriers B;
  __shared__ Piece piece_s;
  __shared__ uint32_t tmem_slot;
  __shared__ int bad_pages[2];                          // in units that the CTA begins, in one that it goes on with
  __shared__ int abort_flag, counted[kChThreads / 32];
  __shared__ float step_max[2][2][kFetchWarps];         // [tile & 1][K, V][warp]
  __shared__ volatile float k_factor[kInfo], v_shift[kInfo];   // per tile: the logits' factor, log2 of the weights'
  __shared__ volatile float o_factor[2];                // per piece: what O is multiplied with
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t q_at = base, k_at = base + 2 * C::kTileBytesD, v_at = base + 4 * C::kTileBytesD;
  const uint32_t q_thin = base + 6 * C::kTileBytesD, k_thin = q_thin + 2 * kThinBytes;
  auto wait = [&](uint64_t* bar, int phase) { return mbar_wait(bar, (uint32_t)phase & 1u, &abort_flag, c.dev_status, kDevTimeout, a.wait_limit); };

  if (threadIdx.x == 0) {
    abort_flag = bad_pages[0] = bad_pages[1] = 0;
    for (int i = 0; i < 2; ++i) {
      mbar_init(&B.q_full[i], 128);
      for (int half = 0; half < 2; ++half) {
        mbar_init(&B.s_full[i][half], 1);
        mbar_init(&B.p_full[i][half], 128);
        mbar_init(&B.pv_done[i][half], 1);
      }
      mbar_init(&B.k_full[i], kFetch);
      mbar_init(&B.k_empty[i], 1);
      mbar_init(&B.v_full[i], kFetch);
      mbar_init(&B.v_empty[i], 1);
    }
    mbar_init(&B.drained, 1);
    fence_mbar_init();
  }
  if (warp == kSoftmaxWarps + kFetchWarps) {
    tmem_alloc(&tmem_slot, 512);
    tmem_relinquish();
  }
  grid_dependency_wait();
  grid_dependency_launch();
  auto tiles_of = [&](int unit) { return max(1, unit_tiles(c, a.row_tiles, unit)); };   // a unit without rows has its outputs written, too
  {
    // The CTA's run of tiles: every thread counts those of some units; the threads in whose units the run begins and ends say where.
    const int units = c.batch * c.Hkv * a.row_tiles, per = (units + kChThreads - 1) / kChThreads;
    const int u0 = min((int)threadIdx.x * per, units), u1 = min(u0 + per, units);
    int sum = 0;
    for (int u = u0; u < u1; ++u) sum += tiles_of(u);
    int upto = sum, all = 0, first = 0;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const int o = __shfl_up_sync(0xffffffffu, upto, off);
      if (lane >= off) upto += o;
    }
    if (lane == 31) counted[warp] = upto;
    __syncthreads();
#pragma unroll
    for (int x = 0; x < kChThreads / 32; ++x) {
      first += x < warp ? counted[x] : 0;
      all += counted[x];
    }
    first += upto - sum;
    const Deal deal(all, gridDim.x, kChSnap);
    const int x = blockIdx.x;
    if (threadIdx.x == 0) {
      if (x >= deal.ctas) piece_s.run = Run{0, 0, 0, 0, 1};
      else if (x + 1 == deal.ctas) piece_s.run.end = all;
    }
    for (int k = 0; k < 2; ++k) {
      if (x + k >= deal.ctas) break;
      const int want = deal.start(x + k);
      if (want < first || want >= first + sum) continue;
      int u = u0, f = first, t = tiles_of(u);
      while (want >= f + t) {
        f += t;
        t = tiles_of(++u);
      }
      const int boundary = f + deal.moved(want - f, t);
      if (k == 1) {
        piece_s.run.end = boundary;
      } else {
        piece_s.run.tile = boundary;
        piece_s.run.entry = u;
        piece_s.run.first = f;
        piece_s.run.tiles = t;
      }
    }
    __syncthreads();
    if (threadIdx.x == 0) {
      const Run run = piece_s.run;
      if (run.tile < run.end) piece_s.cut(1, tiles_of);
      a.begins[blockIdx.x] = run.tile < run.end ? make_int4(piece_s.unit, piece_s.t0, 0, 0) : make_int4(-1, 0, 0, 0);
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  constexpr uint32_t kO = 256;                          // O of tile w: columns kO + w * kD; S and P: w * 128
  const volatile Piece& piece = piece_s;

  struct Unit {
    int b, h, rho0, n, count, t0, tiles, done, nth;     // done: tiles of the pieces before, phases of the rings; nth: pieces before
  };
  // A role's part of every piece.  All roles go from piece to piece together.
  auto each_piece = [&](auto&& part) {
    int done = 0;
    for (int nth = 0; piece.run.tile < piece.run.end; ++nth) {
    const int unit = piece.unit, bh = unit / a.row_tiles, rho0 = (unit - bh * a.row_tiles) * kChRows, b = bh / c.Hkv, h = bh - b * c.Hkv;
    const int n = paged_length(c, b, h), count = paged_count(c, b), t0 = piece.t0, tiles = min(piece.t1, unit_tiles(c, a.row_tiles, unit)) - t0;
    if (threadIdx.x == 0 && t0 == 0) check_length(c, b, h);
    part(Unit{b, h, rho0, n, count, t0, tiles, done, nth});
    __syncwarp();
    // all go on to the next piece, or none
    const bool stop = __syncthreads_or(abort_flag) != 0;
    tc_fence_after();
    done += tiles;
    if (threadIdx.x == 0) {
      piece_s.run.tile += piece_s.t1 - piece_s.t0;
      if (stop) piece_s.run.tile = piece_s.run.end;
      if (piece_s.run.tile < piece_s.run.end) piece_s.cut(1, tiles_of);
    }
    __syncthreads();
    }
  };

  if (warp >= kSoftmaxWarps && warp < kSoftmaxWarps + kFetchWarps) {
    each_piece([&](const Unit& u) {
      // ---------------- fetching K and V, half a row per thread ----------------
      // Pieces 0 .. 7 are K's: 32 rows, half of their words each; 8 .. 15 V's.  Warp f takes f, f + 7, f + 14.
      const int b = u.b, h = u.h, n = u.n, t0 = u.t0, tiles = u.tiles, done = u.done, nth = u.nth;
      const int fw = warp - kSoftmaxWarps;
      const bool first = threadIdx.x == kSoftmaxWarps * 32;
      constexpr int kPieces = (16 + kFetchWarps - 1) / kFetchWarps, kHalf = 2 * kWords;   // 32-bit words of codes of half a row
      const int per_page = c.page_rows / kBlockRows;
      auto row_of = [&](int x) { return ((fw + x * kFetchWarps) >> 1 & 3) * 32 + lane; };
      auto half_of = [&](int x) { return (fw + x * kFetchWarps) & 1; };
      auto is_v = [&](int x) { return fw + x * kFetchWarps >= 8; };
      auto has = [&](int x) { return fw + x * kFetchWarps < 16; };
      auto page_of = [&](int j, int x) {                // of the thread's row of tile j; -1: nothing there
        const int row = (t0 + j) * kChTile + row_of(x);
        return has(x) && j < tiles && row < n ? c.table[(long long)b * c.table_width + row / c.page_rows] : -1;
      };
      auto place_of = [&](int j, int x, int page) {     // block of the pool, -1
        const int row = (t0 + j) * kChTile + row_of(x);
        if (!has(x) || j >= tiles || row >= n) return -1;
        if ((unsigned int)page >= (unsigned int)c.n_pages) {
          atomicOr(c.dev_status, kDevBadIndex);
          return -1;
        }
        return (page * c.Hkv + h) * per_page + row % c.page_rows / kBlockRows;
      };
      bool ok = true;
      int page[kPieces];
#pragma unroll
      for (int x = 0; x < kPieces; ++x) page[x] = page_of(0, x);
      if constexpr (kInt4) {
        uint32_t codes[kPieces][kHalf], params[kPieces][kG];   // half a row's codes; (step, offset) per group
        unsigned short step_of[kPieces][kG], offset_of[kPieces][kG];
        bool there[kPieces];
        int a_ref = 0;
        auto load = [&](int j) {                        // tile j's, and the next one's pages
#pragma unroll
          for (int x = 0; x < kPieces; ++x) {
            // Rows that are not there read block 0 in their place and have no steps: nothing here waits for what it loads, which a
            // branch around the loads, or steps and offsets put together here, would do once per piece.
            const int place = place_of(j, x, page[x]), q = lane & 15;
            there[x] = place >= 0;
            const bool v = is_v(x);
            const uint8_t* block = (v ? c.V : c.K) + (size_t)(unsigned int)max(place, 0) * (unsigned int)c.block_bytes;
#pragma unroll
            for (int y = 0; y < kHalf / 4; ++y) {
              const uint4 w = reinterpret_cast<const uint4*>(block + q * (kD / 2) + half_of(x) * (kD / 4))[y];
              codes[x][4 * y] = w.x; codes[x][4 * y + 1] = w.y; codes[x][4 * y + 2] = w.z; codes[x][4 * y + 3] = w.w;
            }
#pragma unroll
            for (int g = 0; g < kG; ++g) {
              const unsigned short* p = reinterpret_cast<const unsigned short*>(block + int4_params(kD, g, q));
              step_of[x][g] = p[0];
              offset_of[x][g] = p[4];
            }
          }
#pragma unroll
          for (int x = 0; x < kPieces; ++x) page[x] = page_of(j + 1, x);
        };
        load(0);
        for (int j = 0; j < tiles; ++j) {               // to the end even when a wait ran out: the warps meet in every round
          const int at = done + j, s = at & 1;
          // the tile's exponents: its largest step just below 2^15, its largest offset well within f16
          float most[2] = {0.f, 0.f};
#pragma unroll
          for (int x = 0; x < kPieces; ++x)
#pragma unroll
            for (int g = 0; g < kG; ++g) {
              params[x][g] = there[x] ? step_of[x][g] | (uint32_t)offset_of[x][g] << 16 : 0u;
              const float m = fmaxf(lower(params[x][g]), fabsf(upper(params[x][g])) * (is_v(x) ? 0x1p-25f : 0x1p-16f));
              if (is_v(x)) most[1] = fmaxf(most[1], m);
              else most[0] = fmaxf(most[0], m);
            }
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            const float m = __uint_as_float(__reduce_max_sync(0xffffffffu, __float_as_uint(most[x])));
            if (lane == 0) step_max[s][x][fw] = m;
          }
          fetch_sync();
          float kt = 0x1p-40f, vt = 0x1p-40f;
#pragma unroll
          for (int x = 0; x < kFetchWarps; ++x) { kt = fmaxf(kt, step_max[s][0][x]); vt = fmaxf(vt, step_max[s][1][x]); }
          const int ka = 141 - (int)(__float_as_uint(kt) >> 23), va = 141 - (int)(__float_as_uint(vt) >> 23);
          if (j == 0) a_ref = va;
          if (first) {
            k_factor[at % kInfo] = power_of_two(24 - ka);
            v_shift[at % kInfo] = (float)(a_ref - va);
            if (j == 0) o_factor[nth & 1] = power_of_two(24 - a_ref);
          }
          ok = ok && (at < 2 || wait(&B.k_empty[s], (at >> 1) - 1));
          bool v_free = false;
#pragma unroll
          for (int x = 0; x < kPieces; ++x) {
            if (!has(x)) continue;
            const int r = row_of(x);
            if (!is_v(x)) {
              if (!ok) continue;
#pragma unroll
              for (int g = 0; g < kG; ++g) {
                const float step = lower(params[x][g]) * power_of_two(ka);
                const uint32_t s1 = pack_f16x2(step, step), s16 = pack_f16x2(step * 0.0625f, step * 0.0625f), l = pack_f16x2(step * -0x1p-21f, step * -0x1p-21f);
#pragma unroll
                for (int m = g * kPerGroup; m < (g + 1) * kPerGroup; ++m)
#pragma unroll
                  for (int q = 0; q < 2; ++q)           // word (2 half + q) * kWords + m of the row: dims 32 m + 8 (2 half + q) ..
                    operands_of(codes[x][q * kWords + m], s1, s16, l, operand_at(k_at + (uint32_t)s * C::kTileBytesD, r, 4 * m + 2 * half_of(x) + q));
              }
              if (half_of(x) == 0) {
                uint32_t thin[8] = {0u, 0u, 0u, 0u, 0u, 0u, 0u, 0u};   // dims 3 g ..: hi, lo, hi against sum(q)'s hi, hi, lo
#pragma unroll
                for (int g = 0; g < kG; ++g) {          // times 2^8, as sum(q)'s are times 2^-8
                  const uint32_t mid = split_f16(fmaf(8.f, lower(params[x][g]), upper(params[x][g])) * power_of_two(ka - 16));
#pragma unroll
                  for (int y = 0; y < 3; ++y) {
                    const uint32_t part = y == 1 ? mid >> 16 : mid & 0xFFFFu;
                    thin[(3 * g + y) >> 1] |= (3 * g + y) & 1 ? part << 16 : part;
                  }
                }
                const uint32_t to = thin_at(k_thin + (uint32_t)s * kThinBytes, r);
                sts128(to, thin[0], thin[1], thin[2], thin[3]);
                sts128(to + 128u, thin[4], thin[5], thin[6], thin[7]);
              }
            } else {
              if (!v_free) {                            // the first of V's: K's are done
                fence_proxy_async_smem();
                mbar_arrive(&B.k_full[s]);
                ok = ok && (at < 2 || wait(&B.v_empty[s], (at >> 1) - 1));
                v_free = true;
              }
              if (!ok) continue;
              uint32_t s1[kG], s16[kG], l[kG];
#pragma unroll
              for (int g = 0; g < kG; ++g) {
                const float step = lower(params[x][g]) * power_of_two(va), lo = upper(params[x][g]) * power_of_two(va - 24);
                s1[g] = pack_f16x2(step, step);
                s16[g] = pack_f16x2(step * 0.0625f, step * 0.0625f);
                l[g] = pack_f16x2(lo, lo);
              }
#pragma unroll
              for (int y = 0; y < kHalf; ++y) {         // word y: dims 32 m + 4 r' + (0..3) in its lower half, 32 (m + 1) + .. in its upper
                const int g = 2 * (y % (kWords / 2)) / kPerGroup, g1 = (2 * (y % (kWords / 2)) + 1) / kPerGroup;
                const uint32_t t1 = g == g1 ? s1[g] : __byte_perm(s1[g], s1[g1], 0x5410), t16 = g == g1 ? s16[g] : __byte_perm(s16[g], s16[g1], 0x5410);
                operands_of(codes[x][y], t1, t16, g == g1 ? l[g] : __byte_perm(l[g], l[g1], 0x5410),
                            operand_at(v_at + (uint32_t)s * C::kTileBytesD, r, half_of(x) * kHalf + y));
              }
            }
          }
          fence_proxy_async_smem();
          if (!v_free) mbar_arrive(&B.k_full[s]);
          mbar_arrive(&B.v_full[s]);
          load(j + 1);                                  // the next tile's codes come while the products run
        }
      } else {
        if (first) o_factor[nth & 1] = 1.f;
        // a side of tile j as a group of copies; `page` is that of tile j
        auto fetch = [&](int j, bool v) {
          const int at = done + j, s = at & 1;
          // the wait's verdict is a warp's: places are exchanged by whole warps
          if (j < tiles && at >= 2 && !__all_sync(0xffffffffu, wait(v ? &B.v_empty[s] : &B.k_empty[s], (at >> 1) - 1))) return false;
#pragma unroll
          for (int x = 0; x < kPieces; ++x) {
            if (!has(x) || is_v(x) != v || j >= tiles) continue;
            // a row's half in kD / 16 threads side by side; the places are those of the rows' own threads
            const int own = place_of(j, x, page[x]), per_row = kD / 16, y = half_of(x) * per_row + lane % per_row;
            const uint32_t to = (v ? v_at : k_at) + (uint32_t)s * C::kTileBytesD;
#pragma unroll
            for (int z = 0; z < per_row; ++z) {
              const int r = z * (32 / per_row) + lane / per_row, place = __shfl_sync(0xffffffffu, own, r);
              copy16(operand_at(to, row_of(x) - lane + r, y), (v ? c.V : c.K) + (size_t)(unsigned int)(place >= 0 ? place : 0) * (32u * kD) + (r & 15) * (2 * kD) + 16 * y,
                     place >= 0);
            }
            page[x] = page_of(j + 1, x);
          }
          copy16_commit();
          return true;
        };
        ok = fetch(0, false) && fetch(0, true);
        for (int j = 0; j < tiles && ok; ++j) {
          const int at = done + j, s = at & 1;
          if (first) { k_factor[at % kInfo] = 1.f; v_shift[at % kInfo] = 0.f; }
          copy16_wait<1>();
          fence_proxy_async_smem();
          mbar_arrive(&B.k_full[s]);
          ok = fetch(j + 1, false);                     // (its slot comes free only once this tile is known to be there)
          copy16_wait<1>();
          fence_proxy_async_smem();
          mbar_arrive(&B.v_full[s]);
          ok = ok && fetch(j + 1, true);
        }
        copy16_wait<0>();
      }
    });
  } else if (warp >= kSoftmaxWarps + kFetchWarps) {
    uint32_t drains = 0;
    each_piece([&](const Unit& u) {
      // ---------------- the products, by one thread ----------------
      const int tiles = u.tiles, done = u.done, nth = u.nth;
      {
        // While the others fetch: are all of the piece's pages there?  If not, the merge makes the unit's rows anew.  (Rows left out in the
        // softmax here: 2-5% of every call's time, whichever way.)
        const int row0 = u.t0 * kChTile, row1 = min((u.t0 + tiles) * kChTile, u.n), pages = row1 > row0 ? (row1 - 1) / c.page_rows + 1 : 0;
        bool bad = false;
#pragma unroll 4
        for (int x = row0 / c.page_rows + lane; x < pages; x += 32)
          bad |= (unsigned int)c.table[(long long)u.b * c.table_width + x] >= (unsigned int)c.n_pages;
        if (bad) bad_pages[u.t0 > 0] = 1;
        __syncwarp();
      }
      if (warp == kSoftmaxWarps + kFetchWarps && tiles > 0 && elect_one()) {
        constexpr uint32_t idesc_s = kInt4 ? make_idesc_f16(128, 64, false) : make_idesc_bf16(128, 64, false);
        constexpr uint32_t idesc_o = kInt4 ? make_idesc_f16(128, kD, true) : make_idesc_bf16(128, kD, true);
        // descriptors count 16-byte units
        const uint64_t q0 = kmajor_desc(q_at), k0 = kmajor_desc(k_at), v0 = make_smem_desc(v_at, 16384u, 1024u);
        const uint64_t qt = make_smem_desc_plain(q_thin, 128u, 256u), kt = make_smem_desc_plain(k_thin, 128u, 256u);
        auto qk = [&](int w, int half, int s) {
          const uint64_t a0 = q0 + (uint64_t)(w * (C::kTileBytesD >> 4)), b0 = k0 + (uint64_t)(s * (C::kTileBytesD >> 4) + half * (8192 >> 4));
          const uint32_t to = tmem + (uint32_t)(w * 128 + half * 64);
#pragma unroll
          for (int k = 0; k < kD / 16; ++k) {
            const uint64_t step = (uint64_t)(((uint32_t)(k >> 2) * 16384u + (uint32_t)(k & 3) * 32u) >> 4);
            umma_ss(to, a0 + step, b0 + step, idesc_s, k > 0);
          }
          if constexpr (kInt4)
            umma_ss(to, qt + (uint64_t)(w * (kThinBytes >> 4)), kt + (uint64_t)(s * (kThinBytes >> 4) + half * (2048 >> 4)), idesc_s, true);
          umma_commit(&B.s_full[w][half]);
        };
        bool ok = true;
        for (int x = 0; x < 4 && ok; ++x) {
          if (x < 2) ok = wait(&B.q_full[x], nth) && (x == 1 || wait(&B.k_full[done & 1], done >> 1));
          if (!ok) break;
          tc_fence_after();
          qk(x & 1, x >> 1, done & 1);
        }
        if (ok) umma_commit(&B.k_empty[done & 1]);
        // Steps x = 4 j + 2 half + w: P V of step x, then S of step x + 3, in whose place are the weights that step x - 1 reads.
        for (int x = 0; x <= 4 * tiles && ok; ++x) {
          if (x < 4 * tiles) {
            const int w = x & 1, half = x >> 1 & 1, at = done + (x >> 2), s = at & 1;
            ok = wait(&B.p_full[w][half], at) && ((x & 3) > 0 || wait(&B.v_full[s], at >> 1));
            if (!ok) break;
            tc_fence_after();
            const uint64_t b0 = v0 + (uint64_t)(s * (C::kTileBytesD >> 4) + half * 512);
#pragma unroll
            for (int k = 0; k < 4; ++k)                 // 16 cache rows: 8 columns of P, 2048 bytes of V
              umma_ts(tmem + kO + (uint32_t)w * kD, tmem + (uint32_t)(w * 128 + half * 64 + k * 8), b0 + (uint64_t)(k * 128), idesc_o, x > 1 || k > 0);
            umma_commit(&B.pv_done[w][half]);
            if ((x & 3) == 3) umma_commit(&B.v_empty[s]);
          }
          const int y = x - 1, at1 = done + (y >> 2) + 1;
          if (y >= 0 && y < 4 * (tiles - 1)) {
            ok = ((y & 3) > 0 || wait(&B.k_full[at1 & 1], at1 >> 1)) && wait(&B.pv_done[y & 1][y >> 1 & 1], at1 - 1);
            if (!ok) break;
            tc_fence_after();
            qk(y & 1, y >> 1 & 1, at1 & 1);
            if ((y & 3) == 3) umma_commit(&B.k_empty[at1 & 1]);
          }
        }
        // Nothing may still write tensor memory, or arrive, when the CTA goes, which it does at the end of a piece in which any role's wait
        // ran out, the softmax's for the last products among them.
        umma_commit(&B.drained);
        wait_issued(&B.drained, drains++);
      }
    });
  } else {
    each_piece([&](const Unit& u) {
      // ---------------- softmax: a query row per thread ----------------
      const int b = u.b, h = u.h, rho0 = u.rho0, n = u.n, count = u.count, t0 = u.t0, tiles = u.tiles, done = u.done, nth = u.nth, R = c.n_tokens * c.G;
      const int w = warp >> 2, r = threadIdx.x & 127, rho = rho0 + w * 128 + r, i = rho / c.G, g = rho - i * c.G;
      const bool live = rho < R && i < count;
      const int sees = live ? n - (count - 1 - i) : n;
      const uint32_t row_lane = (uint32_t)(warp & 3) << 21;          // lanes 32 (warp % 4) .. of tensor memory, in bits 16 up
      const uint32_t s_tm = tmem + row_lane + (uint32_t)w * 128u, o_tm = tmem + row_lane + kO + (uint32_t)w * kD;
      float unscale = 1.f;
      if (tiles > 0) {
        // the warp's rows into shared memory, a row in kD / 8 lanes side by side
        constexpr int kLanes = kD / 8, kRowsAtOnce = 32 / kLanes;
        const uint32_t tile = q_at + (uint32_t)w * C::kTileBytesD;
        const int x = lane % kLanes, row0 = (warp & 3) * 32 + lane / kLanes;
        // four rows per lane together: what each of them waits for, loads and shuffles, is on its way for all
#pragma unroll 1
        for (int z0 = 0; z0 < 32; z0 += 4 * kRowsAtOnce) {
          uint4 raw[4];
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            const int rho_z = rho0 + w * 128 + row0 + z0 + y * kRowsAtOnce, i_z = rho_z / c.G, g_z = rho_z - i_z * c.G;
            const __nv_bfloat16* q = reinterpret_cast<const __nv_bfloat16*>(a.Q.data) + b * a.Q.sb + (long long)(h * c.G + g_z) * a.Q.sh + i_z * a.Q.sn;
            raw[y] = rho_z < R && i_z < count ? reinterpret_cast<const uint4*>(q)[x] : make_uint4(0u, 0u, 0u, 0u);
          }
          if constexpr (kInt4) {
            float top[4], sum[4];
#pragma unroll
            for (int y = 0; y < 4; ++y) {
              const uint32_t* u = &raw[y].x;
              top[y] = 0.f;
#pragma unroll
              for (int k = 0; k < 4; ++k) top[y] = fmax3(top[y], fabsf(lower(u[k])), fabsf(upper(u[k])));
            }
#pragma unroll
            for (int off = 1; off < kLanes; off <<= 1)
#pragma unroll
              for (int y = 0; y < 4; ++y) top[y] = fmaxf(top[y], __shfl_xor_sync(0xffffffffu, top[y], off));
#pragma unroll
            for (int y = 0; y < 4; ++y) {
              // 2^e top in [2^14, 2^15), for top of 2^-86 .. 2^100; an infinite one makes the row's logits NaN
              int e = 141 - (int)(__float_as_uint(top[y]) >> 23);
              e = e < -100 ? -100 : e > 100 ? 100 : e;
              const float scale = top[y] < INFINITY ? power_of_two(e) : __uint_as_float(0x7FFFFFFFu);
              // of the rows that the warp's lanes have in turn, each thread keeps its own's
              const float back = __shfl_sync(0xffffffffu, power_of_two(-e), lane % kRowsAtOnce * kLanes);
              if (lane / kRowsAtOnce == z0 / kRowsAtOnce + y) unscale = back;
              float v[8];
              const uint32_t* u = &raw[y].x;
#pragma unroll
              for (int k = 0; k < 4; ++k) {
                v[2 * k] = lower(u[k]) * scale;
                v[2 * k + 1] = upper(u[k]) * scale;
              }
              // dims in the order of K's operands
              sts128(operand_at(tile, row0 + z0 + y * kRowsAtOnce, x), pack_f16x2(v[0], v[4]), pack_f16x2(v[1], v[5]), pack_f16x2(v[2], v[6]), pack_f16x2(v[3], v[7]));
              sum[y] = ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
            }
#pragma unroll
            for (int off = 1; off < kLanes / kG; off <<= 1)
#pragma unroll
              for (int y = 0; y < 4; ++y) sum[y] += __shfl_xor_sync(0xffffffffu, sum[y], off);
            uint32_t parts[4][kG];
#pragma unroll
            for (int g2 = 0; g2 < kG; ++g2)
#pragma unroll
              for (int y = 0; y < 4; ++y) parts[y][g2] = split_f16(__shfl_sync(0xffffffffu, sum[y], lane / kLanes * kLanes + g2 * (kLanes / kG)) * 0x1p-8f);
#pragma unroll
            for (int y = 0; y < 4; ++y) {
              uint32_t thin[8] = {0u, 0u, 0u, 0u, 0u, 0u, 0u, 0u};
#pragma unroll
              for (int g2 = 0; g2 < kG; ++g2)
#pragma unroll
                for (int k = 0; k < 3; ++k) {
                  const uint32_t part = k == 2 ? parts[y][g2] >> 16 : parts[y][g2] & 0xFFFFu;
                  thin[(3 * g2 + k) >> 1] |= (3 * g2 + k) & 1 ? part << 16 : part;
                }
              const uint32_t to = thin_at(q_thin + (uint32_t)w * kThinBytes, row0 + z0 + y * kRowsAtOnce);
              if (x == 0) sts128(to, thin[0], thin[1], thin[2], thin[3]);
              if (x == 1) sts128(to + 128u, thin[4], thin[5], thin[6], thin[7]);
            }
          } else {
#pragma unroll
            for (int y = 0; y < 4; ++y) sts128(operand_at(tile, row0 + z0 + y * kRowsAtOnce, x), raw[y].x, raw[y].y, raw[y].z, raw[y].w);
          }
        }
        fence_proxy_async_smem();
      }
      mbar_arrive(&B.q_full[w]);
      const float factor = (kCap ? c.scale / c.softcap : c.scale * kLog2e) * unscale;   // to the tanh's argument, or to log2 units
      float ref = -INFINITY, l = 0.f;                   // weights are 2^(logit - ref)
      const int sees_all = __reduce_min_sync(0xffffffffu, sees);   // what every row of the warp sees
      bool ok = true;
      for (int j2 = 0; j2 < 2 * tiles; ++j2) {
        const int j = j2 >> 1, half = j2 & 1, at = done + j;
        // the waits' verdict is a warp's: tensor memory is read by whole warps
        ok = ok && __all_sync(0xffffffffu, wait(&B.s_full[w][half], at));
        if (!ok) break;
        tc_fence_after();
        const uint32_t s_half = s_tm + (uint32_t)half * 64u;
        const float f = kCap ? fminf(factor * k_factor[at % kInfo], 0x1p126f) : factor * k_factor[at % kInfo], shift = v_shift[at % kInfo];
        const int left = sees - (t0 + j) * kChTile - half * 64;     // columns that the row sees
        const bool edge = sees_all < (t0 + j) * kChTile + half * 64 + 64;
        // One pass: the weights of 32 columns at a time by the reference as it stands.  Where a row's logits have outgrown it, its sums, O and
        // what this half has of P so far are scaled down first (the first tile's reference comes about so, too).
        const float to_log2 = kCap ? c.softcap * kLog2e : f;
        const f32x2 ff = f2_make(f, f), f1 = f2_make(to_log2, to_log2);
        const float to_l = ex2_approx(-shift);
        float v[64];
        for (;;) {
          tmem_ld32(s_half, v);
          tmem_ld32(s_half + 32u, v + 32);
          tmem_wait_ld();
          if constexpr (kCap) {
            float far0 = 0.f, far1 = 0.f;
#pragma unroll
            for (int y = 0; y < 64; y += 4) {
              far0 = fmax3(far0, fabsf(v[y]), fabsf(v[y + 1]));
              far1 = fmax3(far1, fabsf(v[y + 2]), fabsf(v[y + 3]));
            }
            if (__all_sync(0xffffffffu, fmaxf(far0, far1) * f <= kTanhNear)) {
#pragma unroll
              for (int y = 0; y < 64; y += 2) {
                const f32x2 z = tanh_near(f2_mul(f2_make(v[y], v[y + 1]), ff));
                v[y] = f2_lo(z);
                v[y + 1] = f2_hi(z);
              }
            } else if (c.softcap <= kTanhFarAlone) {
#pragma unroll
              for (int y = 0; y < 64; ++y) v[y] = tanh_far(v[y] * f);
            } else {
#pragma unroll
              for (int y = 0; y < 64; y += 2) {
                v[y] *= f;
                v[y + 1] *= f;
                tanh_any(v[y], v[y + 1]);
              }
            }
          }
          if (edge) {
#pragma unroll
            for (int y = 0; y < 64; ++y)
              if (y >= left) v[y] = -INFINITY;
          }
          float m[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
          for (int y = 4; y < 60; y += 8)
#pragma unroll
            for (int z = 0; z < 4; ++z) m[z] = fmax3(m[z], v[y + 2 * z], v[y + 2 * z + 1]);
          m[0] = fmax3(m[0], v[60], v[61]);
          m[1] = fmax3(m[1], v[62], v[63]);
          const float mx = fmaf(fmaxf(fmax3(m[0], m[1], m[2]), m[3]), to_log2, shift);   // (the factor is positive)
          if (!__any_sync(0xffffffffu, mx > ref + kChSlack)) break;
          float down = 1.f;
          if (mx > ref + kChSlack) {
            const float next = ceilf(mx) - kChStart;
            down = ex2_approx(ref - next);              // ref = -inf gives 0
            ref = next;
          }
          l *= down;
          if (j2 > 0) {                                 // the products of the half before may still be adding to O
            ok = __all_sync(0xffffffffu, wait(&B.pv_done[w][half ^ 1], half ? at : at - 1));
            tc_fence_after();
            if (ok) rescale(o_tm, kD, down);
          }                                             // (then the logits again: kept across the call, each would be copied every time)
        }
        const float m_use = (ref == -INFINITY ? 0.f : ref) - shift;   // only logits of -inf so far: they weigh nothing
        const f32x2 minus_m = f2_make(-m_use, -m_use);
        f32x2 sum0 = f2_make(0.f, 0.f), sum1 = sum0;
#pragma unroll
        for (int x = 0; x < 64; x += 32) {
          uint32_t p[16];
#pragma unroll
          for (int y = 0; y < 32; y += 4) {
            const f32x2 a0 = f2_fma(f2_make(v[x + y], v[x + y + 1]), f1, minus_m), a1 = f2_fma(f2_make(v[x + y + 2], v[x + y + 3]), f1, minus_m);
            const float e0 = ex2_approx(f2_lo(a0)), e1 = ex2_approx(f2_hi(a0)), e2 = ex2_approx(f2_lo(a1)), e3 = ex2_approx(f2_hi(a1));
            sum0 = f2_add(sum0, f2_make(e0, e1));
            sum1 = f2_add(sum1, f2_make(e2, e3));
            p[y / 2] = kInt4 ? pack_f16x2(e0, e1) : pack_bf16x2(e0, e1);
            p[y / 2 + 1] = kInt4 ? pack_f16x2(e2, e3) : pack_bf16x2(e2, e3);
          }
          tmem_st16(s_half + x / 2, p);                 // P where S has been read already
        }
        sum0 = f2_add(sum0, sum1);
        l = fmaf(f2_lo(sum0) + f2_hi(sum0), to_l, l);
        tmem_wait_st();
        tc_fence_before();
        mbar_arrive(&B.p_full[w][half]);
      }
      // ---- the row's result ----
      if (ok && tiles > 0) ok = __all_sync(0xffffffffu, wait(&B.pv_done[w][1], done + tiles - 1));
      if (ok) {
        tc_fence_after();
        const bool whole = piece.whole != 0, some = l > 0.f && live;
        const float ofac = tiles > 0 ? o_factor[nth & 1] : 0.f, norm = whole ? (some ? ofac / l : 0.f) : ofac;
        const bool nothing = tiles == 0 || (whole && !some);
        float* const part = a.part + (long long)(2 * blockIdx.x + (t0 == 0)) * kChRows * (kD + 2);
        const long long row = ((long long)b * c.Hq + h * c.G + g) * c.n_tokens + i;
        // By way of the warp's rows of Q's tile, which no product reads any more, for stores of whole rows: kD values of 16 bits at once,
        // or fp32 ones in two turns.  16-byte chunk k of row r is at k ^ r.
        constexpr int kChunks = kD / 8;
        const uint32_t staged = q_at + (uint32_t)w * C::kTileBytesD + (uint32_t)(warp & 3) * (32u * 2u * kD);
        const uint32_t mine = staged + (uint32_t)lane * (2u * kD);
        for (int turn = 0; turn < (whole ? 1 : 2); ++turn) {
          auto emit = [&](int dim, float x0, float x1, float x2, float x3) {
            if (nothing) x0 = x1 = x2 = x3 = 0.f;
            if (whole) {
              const uint32_t to = mine + (uint32_t)(((dim / 8) ^ (lane & (kChunks - 1))) * 16 + (dim & 4) * 2);
              asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(to), "r"(pack_bf16x2(x0 * norm, x1 * norm)), "r"(pack_bf16x2(x2 * norm, x3 * norm)) : "memory");
            } else if (dim / (kD / 2) == turn) {
              sts128(mine + (uint32_t)(((dim % (kD / 2) / 4) ^ (lane & (kChunks - 1))) * 16), __float_as_uint(x0 * norm), __float_as_uint(x1 * norm),
                     __float_as_uint(x2 * norm), __float_as_uint(x3 * norm));
            }
          };
#pragma unroll
          for (int x = 0; x < kD / 32; ++x) {
            float v[32];
            if (tiles > 0) {
              tmem_ld32(o_tm + x * 32, v);
              tmem_wait_ld();
            } else {
#pragma unroll
              for (int y = 0; y < 32; ++y) v[y] = 0.f;
            }
#pragma unroll
            for (int y = 0; y < 4; ++y) {
              const float* o = v + 8 * y;
              if constexpr (kInt4) {                    // chunk k of V's operand: dims 32 m + 4 r' + (0..3) and 32 (m + 1) + 4 r' + (0..3) in turn
                const int k = 4 * x + y, dim = 4 * (k / (kWords / 2)) + 64 * (k % (kWords / 2));
                emit(dim, o[0], o[2], o[4], o[6]);
                emit(dim + 32, o[1], o[3], o[5], o[7]);
              } else {
                emit(32 * x + 8 * y, o[0], o[1], o[2], o[3]);
                emit(32 * x + 8 * y + 4, o[4], o[5], o[6], o[7]);
              }
            }
          }
          __syncwarp();
          const int k = lane % kChunks, in_tile = w * 128 + (warp & 3) * 32;
#pragma unroll 4
          for (int z = 0; z < 32; z += 32 / kChunks) {
            const int at = z + lane / kChunks;
            const long long to = __shfl_sync(0xffffffffu, row, at);
            if (rho0 + in_tile + at >= R) continue;
            const uint4 u = lds128(staged + (uint32_t)at * (2u * kD) + (uint32_t)((k ^ (at & (kChunks - 1))) * 16));
            if (whole) reinterpret_cast<uint4*>(a.out + to * kD)[k] = u;
            else reinterpret_cast<uint4*>(part + (in_tile + at) * kD + turn * (kD / 2))[k] = u;
          }
          __syncwarp();
        }
        if (rho < R) {
          if (whole) {
            if (a.lse) a.lse[row] = some ? fmaf(ref, 0.6931471805599453f, logf(l)) : -INFINITY;
          } else {
            reinterpret_cast<float2*>(a.part + (long long)(2 * blockIdx.x + (t0 == 0)) * kChRows * (kD + 2) + kChRows * kD)[w * 128 + r] = make_float2(ref, l);
          }
        }
        tc_fence_before();
      }
    });
  }
  __syncthreads();
  if (threadIdx.x == 0 && (bad_pages[0] | bad_pages[1]) != 0) {
    a.begins[blockIdx.x].z = bad_pages[0];
    a.begins[blockIdx.x].w = bad_pages[1];
  }
  if (warp == kSoftmaxWarps + kFetchWarps) tmem_dealloc(tmem, 512);
}

// Query row rho of a KV head by one warp in fp32, without the rows of bad pages: for units that have some, a call that reports an error.
template <int kD, bool kInt4>
__device__ __noinline__ void row_past_bad_pages(const PagedMmaArgs& a, int unit, int row) {
  const PagedCache& c = a.c;
  const int bh = unit / a.row_tiles, b = bh / c.Hkv, h = bh - b * c.Hkv, rho = (unit - bh * a.row_tiles) * kChRows + row;
  if (rho >= c.n_tokens * c.G) return;
  constexpr int kLanes = kD / 8, kAtOnce = 32 / kLanes;      // 8 dims of a cache row per lane
  const int lane = threadIdx.x & 31, chunk = lane % kLanes, i = rho / c.G, g = rho - i * c.G, count = paged_count(c, b);
  const int sees = i < count ? paged_length(c, b, h) - (count - 1 - i) : 0;
  float q[8], k[8], v[8], m = -INFINITY, l = 0.f, o[8] = {};
  Pack8<__nv_bfloat16> raw;
  raw.load(reinterpret_cast<const __nv_bfloat16*>(a.Q.data) + b * a.Q.sb + (long long)(h * c.G + g) * a.Q.sh + i * a.Q.sn + chunk * 8);
  raw.get(q);
  for (int r0 = 0; r0 < sees; r0 += kAtOnce) {               // (a block's 16 rows are a multiple of kAtOnce)
    const long long at = paged_block(c, b, h, r0 / kBlockRows);
    if (at < 0) continue;
    const int r = r0 + lane / kLanes;
    load_chunk<__nv_bfloat16, kInt4>(c, c.K + at, r % kBlockRows, chunk, true, k);
    load_chunk<__nv_bfloat16, kInt4>(c, c.V + at, r % kBlockRows, chunk, false, v);
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) s = fmaf(q[e], k[e], s);
#pragma unroll
    for (int off = 1; off < kLanes; off <<= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
    if (r >= sees) continue;                                 // (its row of the page may hold anything)
    s *= c.scale;
    if (c.softcap > 0.f) s = c.softcap * tanhf(s / c.softcap);
    s *= kLog2e;
    const float top = fmaxf(m, s), down = m == -INFINITY ? 0.f : ex2_approx(m - top), p = top == -INFINITY ? 0.f : ex2_approx(s - top);
    m = top;
    l = fmaf(l, down, p);
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = fmaf(o[e], down, p * v[e]);
  }
  __syncwarp();
#pragma unroll
  for (int off = kLanes; off < 32; off <<= 1) {
    const float mo = __shfl_xor_sync(0xffffffffu, m, off), lo = __shfl_xor_sync(0xffffffffu, l, off), top = fmaxf(m, mo);
    const float fa = m == -INFINITY ? 0.f : ex2_approx(m - top), fb = mo == -INFINITY ? 0.f : ex2_approx(mo - top);
    l = l * fa + lo * fb;
#pragma unroll
    for (int e = 0; e < 8; ++e) o[e] = o[e] * fa + __shfl_xor_sync(0xffffffffu, o[e], off) * fb;
    m = top;
  }
  if (lane >= kLanes) return;
  const float x[2][4] = {{o[0], o[1], o[2], o[3]}, {o[4], o[5], o[6], o[7]}};
  write_row<kD, 4>(a, b, h, rho, count, 2 * chunk, x[0], m, l);
  write_row<kD, 4>(a, b, h, rho, count, 2 * chunk + 1, x[1], m, l);
}

// grid (CTAs of the kernel before, 32), block 256: merges what several of them left of a unit, a row per warp.  A unit is merged by the
// blocks of the first CTA that began inside it.  Units with bad pages are made anew: those of several CTAs there, others by the blocks of theirs.
template <int kD, bool kInt4>
__global__ void __launch_bounds__(256) paged_chunk_combine_kernel(const __grid_constant__ PagedMmaArgs a) {
  grid_dependency_wait();
  grid_dependency_launch();
  const PagedCache& c = a.c;
  const int x = blockIdx.x, ctas = gridDim.x, lane = threadIdx.x & 31;
  const int4 mine = __ldcg(a.begins + x);
  const int row = (int)blockIdx.y * 8 + (threadIdx.x >> 5);
  if (mine.z != 0) {
    const int next = x + 1 < ctas ? __ldcg(a.begins + x + 1).x : -1;
    for (int u = mine.y == 0 ? mine.x : mine.x + 1; u < (next < 0 ? c.batch * c.Hkv * a.row_tiles : next); ++u) row_past_bad_pages<kD, kInt4>(a, u, row);
  }
  if (mine.x < 0 || mine.y == 0) return;                // (the first CTA begins a unit: x > 0 from here on)
  int bad = 0;                                          // of the pieces that this lane looks at
  auto inside = [&](int y) {
    const int4 o = __ldcg(a.begins + y);
    const bool is = o.x == mine.x && o.y > 0;
    if (is) bad |= o.w;
    return is;
  };
  if (inside(x - 1)) return;
  if (lane == 0) bad |= __ldcg(a.begins + x - 1).z;     // (or of another unit that it begins)
  const int unit = mine.x, bh = unit / a.row_tiles, b = bh / c.Hkv, h = bh - b * c.Hkv, count = paged_count(c, b);
  const int rho = (unit - bh * a.row_tiles) * kChRows + row;
  if (rho >= c.n_tokens * c.G) return;
  constexpr long long kSlot = kChRows * (kD + 2);
  constexpr int kPer = kD / 32;
  auto piece = [&](int k) { return a.part + (2ll * (x - 1 + k) + (k == 0)) * kSlot; };   // the CTA before began the unit
  // 32 pieces at a time, a lane's (reference, sum) each
  float mm = -INFINITY, ll = 0.f, acc[kPer] = {};
  for (int base = 0;; base += 32) {
    const int k = base + lane;
    const bool some = k == 0 || (x - 1 + k < ctas && inside(x - 1 + k));
    const int n = __popc(__ballot_sync(0xffffffffu, some));
    const float2 ml = some ? __ldcg(reinterpret_cast<const float2*>(piece(k) + kChRows * kD) + row) : make_float2(-INFINITY, 0.f);
    float top = ml.x;
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, off));
    top = fmaxf(top, mm);
    const float down = mm == -INFINITY ? 0.f : ex2_approx(mm - top), f = ml.x == -INFINITY ? 0.f : ex2_approx(ml.x - top);
    mm = top;
    float sum = ml.y * f;
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
    ll = fmaf(ll, down, sum);
#pragma unroll
    for (int y = 0; y < kPer; ++y) acc[y] *= down;
#pragma unroll 8
    for (int y = 0; y < n; ++y) {
      const float g = __shfl_sync(0xffffffffu, f, y);
      const float* o = piece(base + y) + row * kD + kPer * lane;
      float w[kPer];
      if constexpr (kPer == 4) {
        const float4 u = __ldcg(reinterpret_cast<const float4*>(o));
        w[0] = u.x; w[1] = u.y; w[2] = u.z; w[3] = u.w;
      } else {
        const float2 u = __ldcg(reinterpret_cast<const float2*>(o));
        w[0] = u.x; w[1] = u.y;
      }
#pragma unroll
      for (int z = 0; z < kPer; ++z) acc[z] = g > 0.f ? fmaf(w[z], g, acc[z]) : acc[z];
    }
    if (n < 32) break;
  }
  if (__any_sync(0xffffffffu, bad)) {
    row_past_bad_pages<kD, kInt4>(a, unit, row);
    return;
  }
  write_row<kD, kPer>(a, b, h, rho, count, lane, acc, mm, ll);
}

struct ChunkVariant {
  void (*kernel)(PagedMmaArgs);
  void (*combine)(PagedMmaArgs);
  size_t smem;
};
template <int kD, int kGroups> ChunkVariant chunk_variant(bool cap) {
  return ChunkVariant{cap ? paged_chunk_kernel<kD, kGroups, true> : paged_chunk_kernel<kD, kGroups, false>, paged_chunk_combine_kernel<kD, (kGroups > 0)>, ChunkConfig<kD, kGroups>::kSmem};
}
bool pick_chunk(const PagedCache& c, ChunkVariant* v) {
  const int groups = c.format == RESTKV_PAGES_INT4 ? c.d / c.group : 0;
  switch (c.d * 16 + groups) {
    case 64 * 16 + 0: *v = chunk_variant<64, 0>(c.softcap > 0.f); return true;
    case 64 * 16 + 1: *v = chunk_variant<64, 1>(c.softcap > 0.f); return true;
    case 64 * 16 + 2: *v = chunk_variant<64, 2>(c.softcap > 0.f); return true;
    case 128 * 16 + 0: *v = chunk_variant<128, 0>(c.softcap > 0.f); return true;
    case 128 * 16 + 1: *v = chunk_variant<128, 1>(c.softcap > 0.f); return true;
    case 128 * 16 + 2: *v = chunk_variant<128, 2>(c.softcap > 0.f); return true;
    case 128 * 16 + 4: *v = chunk_variant<128, 4>(c.softcap > 0.f); return true;
    default: return false;
  }
}
int chunk_ctas(int sm_count) { return sm_count < kMaxCtas ? sm_count : kMaxCtas; }

}  // namespace

cudaError_t paged_chunk_init() {
  PagedCache c{};
  for (float cap : {0.f, 1.f})
    for (int d : {64, 128})
      for (int group : {0, 32, 64, 128}) {
        c.d = d; c.group = group; c.softcap = cap;
        c.format = group ? RESTKV_PAGES_INT4 : RESTKV_PAGES_BF16;
        ChunkVariant v;
        if (group > d || !pick_chunk(c, &v)) continue;
        const cudaError_t e = cudaFuncSetAttribute(v.kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)v.smem);
        if (e != cudaSuccess) return e;
      }
  return cudaSuccess;
}

bool paged_chunk_shape(const PagedCache& c) {
  ChunkVariant v;
  const long long rows = (long long)c.n_tokens * c.G;
  return rows >= kChunkRows && rows * c.batch * c.Hkv >= kChunkAll && pick_chunk(c, &v);
}

bool paged_chunk_supported(const PagedCache& c) {
  if (!paged_chunk_shape(c)) return false;
  const long long rows = (long long)c.n_tokens * c.G;
  const long long units = (long long)c.batch * c.Hkv * ((rows + kChRows - 1) / kChRows);
  return (c.capacity() / kChTile + 1) * units <= 0x7FFFFFFFll;   // tiles are counted in 32 bits
}

size_t paged_chunk_bytes(const PagedCache& c, int sm_count) {
  return (size_t)chunk_ctas(sm_count) * (2 * kChRows * (c.d + 2) * sizeof(float) + sizeof(int4));
}

cudaError_t launch_paged_chunk(const PagedCache& c, const RowsView& Q, void* out, float* lse, float* part, int sm_count, long long wait_limit,
                               cudaStream_t st) {
  ChunkVariant v;
  if (!pick_chunk(c, &v)) return cudaErrorInvalidValue;
  PagedMmaArgs a{};
  a.c = c; a.Q = Q; a.out = (__nv_bfloat16*)out; a.lse = lse; a.part = part; a.wait_limit = wait_limit;
  a.row_tiles = (int)(((long long)c.n_tokens * c.G + kChRows - 1) / kChRows);
  const int ctas = chunk_ctas(sm_count);
  a.begins = reinterpret_cast<int4*>(part + (size_t)2 * ctas * kChRows * (c.d + 2));
  const cudaError_t e = launch_chained(v.kernel, dim3((unsigned int)ctas), kChThreads, v.smem, st, a);
  if (e != cudaSuccess) return e;
  return launch_chained(v.combine, dim3((unsigned int)ctas, kChRows / 8), 256, 0, st, a);
}

}  // namespace restkv
