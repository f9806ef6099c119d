// Cross attention of many query rows of a KV head (a decoder's prompt, or the tokens of many hypotheses) on tcgen05: bf16, head_dim 64 or 128.
//
// What bounds it: 4 * 128 * 128 * head_dim operations per 128 query rows and 128 rows of K and V are 1024 cycles of the tensor pipe at head_dim 128, and the
// exponentials as many of the special-function unit; between the two the chain logits -> maximum -> exponentials -> weights -> products -> next
// logits, each arrow some 200 cycles of barriers besides.  So
//   - a CTA per SM takes 256 query rows (hypotheses x tokens x heads of the group) in two tiles of 128, each with a warpgroup of its own, a thread per
//     row; a tile of K and V serves both;
//   - K and V come by TMA from where they lie (four dimensions with strides) into a ring of tiles, in the order in which they are used;
//   - a tile of logits is two halves of 64 columns in turn: while a row's thread is at one, the other's weights meet V and its next logits are made (whole
//     tiles in turn, in registers as a whole: 296 us for 283);
//   - the two warpgroups take turns at the exponentials: both at them together would wait for their products together (291 us);
//   - S (fp32) and O of both tiles fill the tensor memory's 512 columns at head_dim 128; P (bf16) takes S's place and is the A operand of P V there;
//   - a thread issues the logits' products, one for each tile the others, so that none waits for what it need not;
//   - every role goes through the pieces of the CTA's run by itself;
//   - the reference of the weights is moved (sums and O scaled) only where they would pass 2^8;
//   - weights are rounded to one bf16, by 2^-8 of each at most, for the product with V (their sum is that of the unrounded ones): outputs are off by 2.3e-3 of
//     their size, 1.65e-3 of which is their own rounding.  A second part, as the kernel of few query rows has, would be half as many products again;
//   - rows behind a source's length: their logits are replaced, and what V holds there is cleared in the last 16 rows that a product reads, for a
//     weight of 0 is to find a number.
// The tiles of all units (source, KV head, 256 query rows) end to end are dealt out evenly; what several CTAs share is merged by a second kernel.
#include <math.h>

#include <type_traits>

#include "cross_tc.cuh"
#include "paged_deal.cuh"

namespace restkv {

namespace {

constexpr int kMaRows = 256;                 // query rows of a unit
constexpr int kMaTile = 128;                 // rows of K and V of a tile
constexpr int kMaSoftmax = 8;                // warps
constexpr int kMaThreads = (kMaSoftmax + 4) * 32;   // the loader, the logits' products, and a warp for each tile's other products
// Registers per thread: of the launch, and as the warpgroups of the softmax and the other one then share them.
constexpr int kMaRegs = 168, kMaSoftmaxRegs = 176, kMaOtherRegs = 152;
static_assert(2 * kMaSoftmaxRegs + kMaOtherRegs == 3 * kMaRegs, "more than the launch has would be waited for");
// Tiles that a CTA could go through while it ends one unit and begins another: each unit counts for as many more, ahead of its own, and a boundary that
// lies nearer to a unit's end moves there.  (8 sources of up to 509 tokens: 4 and 2 108 us, 4 and 8 113, 4 and 1 109, 2 and 2 111.)
constexpr int kMaAhead = 4, kMaSnap = 2;
// Of these a CTA has at least, for what each leaves is merged.  (One source, 8 KV heads of 128, 240 query rows, 2000 rows: 4 26.7 us, 8 32.6;
// 4 sources of 4000: 47.1, 43.0; of 300: 22.1, 27.4.)
constexpr int kMaLeast = 4;
constexpr int kMaEmpty = 2;                  // what a unit without tiles counts for: zeros are written
constexpr float kMaSlack = 8.f;              // log2 of what weights may grow to before O is rescaled

struct CrossManyArgs {
  CrossProblem c;
  float* part;                               // per CTA two of: o [d / 4, 256, 4], (m, l) [256]
  int2* begins;                              // per CTA: unit and tile of it that it begins with; -1: none
  unsigned int* dev_status;
  int row_tiles;                             // units per KV head
  long long wait_limit;
};

template <int kD> struct ManyConfig {
  static constexpr uint32_t kTileBytesD = 128u * kD * 2u;
  static constexpr int kSlots = kD == 128 ? 5 : 8;                       // of the ring: tiles of K and of V in turn
  static constexpr size_t kSmem = (2 + kSlots) * (size_t)kTileBytesD + 1024;
};

struct ManyBarriers {
  uint64_t q_full[2], q_free[2], s_full[2][2], p_full[2][2], pv_done[2][2], full[8], empty[8], turn[2], edge, drained[3];
};

// Row `row`, 16-byte chunk `chunk` of a 16-bit operand tile of 128 rows: boxes of [128 rows x 64 elements], 128-byte swizzle.
__device__ __forceinline__ uint32_t many_at(uint32_t tile, int row, int chunk) {
  return tile + (uint32_t)(chunk >> 3) * 16384u + (uint32_t)row * 128u + (uint32_t)(((chunk & 7) ^ (row & 7)) << 4);
}
__device__ __forceinline__ void many_sts128(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

__device__ __forceinline__ void warp_arrive(uint64_t* bar) {
  __syncwarp();
  if ((threadIdx.x & 31) == 0) mbar_arrive(bar);
}

// Tiles of a unit: none if its source has no rows, or if none of its tokens is there.
__device__ __forceinline__ int many_tiles(const CrossProblem& c, int row_tiles, int unit) {
  const int bh = unit / row_tiles, rho0 = (unit - bh * row_tiles) * kMaRows, b = bh / c.Hkv, n = cross_length(c, b, bh - b * c.Hkv);
  if (n == 0) return 0;
  if (c.counts) {
    const int R = (int)c.rows(), last = (min(rho0 + kMaRows, R) - 1) / c.G;
    bool live = false;
    for (int x = rho0 / c.G; x <= last && !live; x += c.n_tokens - x % c.n_tokens)   // the first of the unit's tokens of every hypothesis
      live = x % c.n_tokens < c.counts[b * c.beams + x / c.n_tokens];
    if (!live) return 0;
  }
  return (n + kMaTile - 1) / kMaTile;
}

template <int kD>
__global__ void __launch_bounds__(kMaThreads, 1)
cross_many_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV, const __grid_constant__ CrossManyArgs a) {
  using C = ManyConfig<kD>;
  constexpr int kSlots = C::kSlots;
  const CrossProblem& c = a.c;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) ManyBarriers B;
  __shared__ Piece piece_s;
  __shared__ uint32_t tmem_slot;
  __shared__ int abort_flag, counted[kMaThreads / 32];
  __shared__ int2 counted_some[kMaThreads / 32];     // units with tiles, and the most of one
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  const uint32_t q_at = base, ring_at = base + 2 * C::kTileBytesD;
  auto wait = [&](uint64_t* bar, int phase) { return mbar_wait<0>(bar, (uint32_t)phase & 1u, &abort_flag, a.dev_status, kDevTimeout, a.wait_limit); };

  if (threadIdx.x == 0) {
    abort_flag = 0;
    for (int i = 0; i < 2; ++i) {
      mbar_init(&B.q_full[i], 4);                       // an arrival per warp: those of 128 threads take hundreds of cycles
      mbar_init(&B.q_free[i], 4);
      mbar_init(&B.turn[i], 4);
      for (int half = 0; half < 2; ++half) {
        mbar_init(&B.s_full[i][half], 1);
        mbar_init(&B.p_full[i][half], 4);
        mbar_init(&B.pv_done[i][half], 1);
      }
    }
    for (int i = 0; i < kSlots; ++i) {
      mbar_init(&B.full[i], 1);
      mbar_init(&B.empty[i], 2);                        // the products of both tiles
    }
    mbar_init(&B.edge, 1);
    for (int i = 0; i < 3; ++i) mbar_init(&B.drained[i], 1);
    fence_mbar_init();
  }
  if (warp == kMaSoftmax + 1) {
    tmem_alloc(&tmem_slot, 512);
    tmem_relinquish();
  }
  if (threadIdx.x == kMaSoftmax * 32) {
    prefetch_tensormap(&tmK);
    prefetch_tensormap(&tmV);
  }
  grid_dependency_wait();
  grid_dependency_launch();
  int ahead = kMaAhead;
  auto counted_of = [&](int tiles) { return tiles > 0 ? ahead + tiles : kMaEmpty; };
  auto tiles_of = [&](int unit) { return counted_of(many_tiles(c, a.row_tiles, unit)); };
  {
    // The CTA's run of tiles: every thread counts those of some units; the threads in whose units the run begins and ends say where.
    const int units = c.sources * c.Hkv * a.row_tiles, per = (units + kMaThreads - 1) / kMaThreads;
    const int u0 = min((int)threadIdx.x * per, units), u1 = min(u0 + per, units);
    int sum = 0, with_some = 0, longest = 0;
    for (int u = u0; u < u1; ++u) {
      const int tiles = many_tiles(c, a.row_tiles, u);
      sum += counted_of(tiles);
      with_some += tiles > 0;
      longest = max(longest, tiles);
    }
    int upto = sum, all = 0, first = 0, some = 0;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const int o = __shfl_up_sync(0xffffffffu, upto, off);
      if (lane >= off) upto += o;
    }
    if (lane == 31) counted[warp] = upto;
    with_some = (int)__reduce_add_sync(0xffffffffu, (unsigned int)with_some);
    longest = (int)__reduce_max_sync(0xffffffffu, (unsigned int)longest);
    if (lane == 0) counted_some[warp] = make_int2(with_some, longest);
    __syncthreads();
#pragma unroll
    for (int x = 0; x < kMaThreads / 32; ++x) {
      first += x < warp ? counted[x] : 0;
      all += counted[x];
      some += counted_some[x].x;
      longest = max(longest, counted_some[x].y);
    }
    first += upto - sum;
    int ctas = min((int)gridDim.x, max(max(1, some), all / kMaLeast));
    if (some == units && units <= ctas && (long long)longest * units == all - (long long)kMaAhead * units) {
      // All of one length: as many CTAs to each, if their shares are about as long as those of all CTAs, of which most would begin two units.
      // (8 sources of 1000 rows, 660 query rows of 4 KV heads: 40.4 -> 29.7 us; of 450 28.4 -> 22.3; one source 29.3, 29.9.)
      const int each = max(1, min(ctas / units, longest / kMaLeast));
      if ((longest + each - 1) / each <= all / ctas + 1) {
        ctas = each * units;
        ahead = 0;
        all -= kMaAhead * units;
        first -= kMaAhead * u0;
        sum -= kMaAhead * (u1 - u0);
      }
    }
    const Deal deal(all, ctas, kMaSnap);
    const int x = blockIdx.x;
    if (threadIdx.x == 0) {
      if (x >= deal.ctas) piece_s.run = Run{0, 0, 0, 0, 1};
      else if (x + 1 == deal.ctas) piece_s.run.end = all;
    }
    for (int k = 0; k < 2; ++k) {
      if (x + k >= deal.ctas) break;
      const int want = deal.start(x + k);
      if (want < first || want >= first + sum) continue;
      int u = u0, f = first, t = per == 1 ? sum : tiles_of(u);
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
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_slot;
  constexpr uint32_t kO = 256;                          // O of tile w: columns kO + w * kD; S and P: w * 128

  struct Unit {
    int b, h, rho0, n, t0, tiles, nth;                  // nth: pieces before
    // tiles of the pieces before and how many of these have some, and of those of them with a second tile of query rows: the barriers' phases
    int done, begun, done2, begun2;
    bool two, whole;                                    // more than 128 query rows; no other CTA has tiles of the unit
    __device__ int done_of(int w) const { return w ? done2 : done; }
    __device__ int begun_of(int w) const { return w ? begun2 : begun; }
  };
  // A role's part of every piece, as long as its waits do not run out.  Every role goes through the pieces by itself: what one needs of another
  // it waits for at a barrier, so that K, V and the first logits of a piece are under way while the results of the one before are written.
  const Run run = piece_s.run;
  auto each_piece = [&](auto&& part) {
    int done = 0, begun = 0, done2 = 0, begun2 = 0, nth = 0, unit = run.entry, from = run.tile - run.first, left = run.end - run.tile;
    if (left > 0 && from >= run.tiles) {                // (the run begins with the unit after)
      from = 0;
      ++unit;
    }
    int tiles = left > 0 ? many_tiles(c, a.row_tiles, unit) : 0;
    if (threadIdx.x == 0) a.begins[blockIdx.x] = tiles > 0 && from + left > ahead ? make_int2(unit, max(0, from - ahead)) : make_int2(-1, 0);
    while (left > 0) {
      const int to = min(from + left, counted_of(tiles)), bh = unit / a.row_tiles, b = bh / c.Hkv, h = bh - b * c.Hkv;
      const int t0 = tiles > 0 ? max(0, from - ahead) : 0, t1 = tiles > 0 ? to - ahead : 0;
      // (a run that ends ahead of a unit's tiles leaves it to the next CTA; one without tiles is its who has its beginning)
      if (tiles > 0 ? t1 > 0 : from == 0) {
        const int rho0 = (unit - bh * a.row_tiles) * kMaRows;
        const bool two = rho0 + 128 < (int)c.rows();
        if (!part(Unit{b, h, rho0, cross_length(c, b, h), t0, t1 - t0, nth, done, begun, done2, begun2, two, t0 == 0 && t1 == tiles})) break;
        done += t1 - t0;
        begun += t1 > t0;
        done2 += two ? t1 - t0 : 0;
        begun2 += two && t1 > t0;
        ++nth;
      }
      left -= to - from;
      from = 0;
      if (left > 0) tiles = many_tiles(c, a.row_tiles, ++unit);
    }
  };

  // descriptors count 16-byte units
  auto there = [&](int x) { return wait(&B.full[x % kSlots], x / kSlots); };
  // ---------------- the logits S = Q K^T, by one thread ----------------
  auto logits = [&]() {
    constexpr uint32_t idesc = make_idesc_bf16(128, 64, false);
    const uint64_t q0 = kmajor_desc(q_at), k0 = kmajor_desc(ring_at);
    auto qk = [&](int s, int w, int half) {
      const uint64_t a0 = q0 + (uint64_t)(w * (C::kTileBytesD >> 4)), b0 = k0 + (uint64_t)(s * (C::kTileBytesD >> 4) + half * (8192 >> 4));
#pragma unroll
      for (int k = 0; k < kD / 16; ++k) {
        const uint64_t step = (uint64_t)(((uint32_t)(k >> 2) * 16384u + (uint32_t)(k & 3) * 32u) >> 4);
        umma_ss(tmem + (uint32_t)(w * 128 + half * 64), a0 + step, b0 + step, idesc, k > 0);
      }
      umma_commit(&B.s_full[w][half]);
    };
    each_piece([&](const Unit& u) {
      bool ok = true;
      for (int j = 0; j < u.tiles && ok; ++j) {
        const int at = u.done + j, s = 2 * at % kSlots;
        ok = there(2 * at);
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const int w = x & 1, half = x >> 1;
          if (w == 1 && !u.two) continue;
          if (j > 0) ok = ok && wait(&B.pv_done[w][half], u.done_of(w) + j - 1);   // in the place of the logits are the weights that the product before reads
          else if (half == 0) ok = ok && wait(&B.q_full[w], u.begun_of(w));
          if (!ok) break;
          tc_fence_after();
          qk(s, w, half);
        }
        if (!ok) break;
        umma_commit(&B.empty[s]);
        umma_commit(&B.empty[s]);                       // (V's tiles have two readers)
      }
      return ok;
    });
    umma_commit(&B.drained[0]);                         // nothing may still write tensor memory, or arrive, when the CTA goes
    wait_issued(&B.drained[0], 0u);
  };
  // ---------------- O += P V of one tile of query rows, by one thread ----------------
  auto outputs = [&](auto tile) {
    constexpr int w = decltype(tile)::value;
    constexpr uint32_t idesc = make_idesc_bf16(128, kD, true);
    const uint64_t v0 = make_smem_desc(ring_at, 16384u, 1024u);
    each_piece([&](const Unit& u) {
      bool ok = true;
      if (w == 1 && !u.two) return true;
      for (int j = 0; j < u.tiles && ok; ++j) {
        const int at = u.done + j, s = (2 * at + 1) % kSlots;
        const int left = u.n - (u.t0 + j) * kMaTile, steps = left >= kMaTile ? 8 : (left + 15) / 16;   // of 16 rows that are there
        const uint64_t b0 = v0 + (uint64_t)(s * (C::kTileBytesD >> 4));
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          // (V's barrier is looked at behind the weights', when the phase before this tile's is known to be over)
          ok = ok && wait(&B.p_full[w][half], u.done_of(w) + j) && (half > 0 || there(2 * at + 1));
          if (!ok) break;
          tc_fence_after();
#pragma unroll
          for (int k = 4 * half; k < 4 * half + 4; ++k)   // 16 rows: 8 columns of P, 2048 bytes of V
            if (k < steps)
              umma_ts(tmem + kO + (uint32_t)w * kD, tmem + (uint32_t)(w * 128 + half * 64 + (k & 3) * 8), b0 + (uint64_t)(k * 128), idesc, j > 0 || k > 0);
          umma_commit(&B.pv_done[w][half]);
        }
        if (ok) umma_commit(&B.empty[s]);
        if (ok && !u.two) umma_commit(&B.empty[s]);     // (for the other tile, which has no rows)
      }
      return ok;
    });
    umma_commit(&B.drained[1 + w]);
    wait_issued(&B.drained[1 + w], 0u);
  };

  // Each side's code sits behind its own register-budget change.
  if (warp >= kMaSoftmax) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kMaOtherRegs));
    if (warp == kMaSoftmax) {
      int edges = 0, asked = 0;                         // tiles asked for
      each_piece([&](const Unit& u) {
        // ---------------- loading K and V, in turn ----------------
        bool ok = true;
        int x = 2 * u.done;
        const int end = x + 2 * u.tiles;
        for (; x < end; ++x) {
          const int s = x % kSlots, row = (u.t0 + ((x - 2 * u.done) >> 1)) * kMaTile;
          // at first no more than a tile of each, ahead of the queries, which all wait for
          if (x == 2) ok = __all_sync(0xffffffffu, wait(&B.q_full[0], u.begun) && (!u.two || wait(&B.q_full[1], u.begun2)));
          if (!ok) break;
          // the verdict is the warp's: it clears rows together
          ok = x < kSlots || __all_sync(0xffffffffu, wait(&B.empty[s], x / kSlots - 1));
          if (!ok) break;
          const bool is_v = x & 1, clear = is_v && u.n < row + kMaTile && (u.n & 15) != 0;
          uint8_t* const to = smem_raw + (ring_at - smem_u32(smem_raw)) + (uint32_t)s * C::kTileBytesD;
          uint64_t* const bar = clear ? &B.edge : &B.full[s];
          if (elect_one()) {
            mbar_arrive_expect_tx(bar, C::kTileBytesD);
#pragma unroll
            for (int y = 0; y < kD / 64; ++y) tma_load_4d(to + y * 16384, is_v ? &tmV : &tmK, bar, y * 64, row, u.h, u.b);
          }
          __syncwarp();
          if (clear) {
            wait_issued(&B.edge, (uint32_t)edges++);      // (a copy that has been asked for comes)
            const int r0 = u.n - row, r1 = (r0 + 15) & ~15;
            for (int y = lane; y < (r1 - r0) * (kD / 8); y += 32) many_sts128(many_at(ring_at + (uint32_t)s * C::kTileBytesD, r0 + y / (kD / 8), y % (kD / 8)), 0u, 0u, 0u, 0u);
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&B.full[s]);
          }
        }
        asked = x;
        return ok;
      });
      // nothing may still be on its way into shared memory when the CTA returns
      for (int y = asked > kSlots ? asked - kSlots : 0; y < asked; ++y) wait_issued(&B.full[y % kSlots], (uint32_t)(y / kSlots));
    } else if (warp == kMaSoftmax + 1) {
      if (elect_one()) logits();
    } else if (warp == kMaSoftmax + 2) {
      if (elect_one()) outputs(std::integral_constant<int, 0>{});
    } else {
      if (elect_one()) outputs(std::integral_constant<int, 1>{});
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kMaSoftmaxRegs));
    each_piece([&](const Unit& u) {
      // ---------------- softmax: a query row per thread ----------------
      const int w = warp >> 2, done = u.done_of(w), tiles = w == 0 || u.two ? u.tiles : 0, R = (int)c.rows();
      const int r = threadIdx.x & 127, rho = u.rho0 + w * 128 + r;
      const uint32_t row_lane = (uint32_t)(warp & 3) << 21;          // lanes 32 (warp % 4) .. of tensor memory, in bits 16 up
      const uint32_t s_tm = tmem + row_lane + (uint32_t)w * 128u, o_tm = tmem + row_lane + kO + (uint32_t)w * kD;
      const CrossRow mine = cross_row(c, u.b, rho < R ? rho : 0);
      const bool live = rho < R && cross_live(c, mine);
      // the rows' place in shared memory, by way of which the other warps may still be writing their results of the piece before
      if (u.nth > 0 && !__all_sync(0xffffffffu, wait(&B.q_free[w], u.nth - 1))) return false;
      if (tiles > 0) {
        // the warp's rows into shared memory, a row in kD / 8 lanes side by side, all of a lane's on their way together
        constexpr int kLanes = kD / 8, kAtOnce = 32 / kLanes, kAhead = 16;
        const uint32_t tile = q_at + (uint32_t)w * C::kTileBytesD;
        const int x = lane % kLanes;
        const long long own = live ? reinterpret_cast<const uint4*>(cross_query<__nv_bfloat16>(c, mine, u.h)) - reinterpret_cast<const uint4*>(c.Q.data) : -1;
#pragma unroll 1
        for (int z0 = 0; z0 < 32; z0 += kAhead * kAtOnce) {
          uint4 raw[kAhead];
#pragma unroll
          for (int y = 0; y < kAhead; ++y) {
            if (z0 + y * kAtOnce >= 32) break;
            const long long from = __shfl_sync(0xffffffffu, own, z0 + y * kAtOnce + lane / kLanes);
            raw[y] = from >= 0 ? reinterpret_cast<const uint4*>(c.Q.data)[from + x] : make_uint4(0u, 0u, 0u, 0u);
          }
#pragma unroll
          for (int y = 0; y < kAhead; ++y) {
            if (z0 + y * kAtOnce >= 32) break;
            many_sts128(many_at(tile, (warp & 3) * 32 + z0 + y * kAtOnce + lane / kLanes, x), raw[y].x, raw[y].y, raw[y].z, raw[y].w);
          }
        }
        fence_proxy_async_smem();
      }
      // (Only where somebody waits for it: nobody may be two phases ahead of who waits for one.)
      if (tiles > 0) warp_arrive(&B.q_full[w]);
      const float f = c.scale * kLog2e;
      float ref = -INFINITY, l = 0.f;                   // weights are 2^(logit - ref)
      bool ok = true;
      for (int j2 = 0; j2 < 2 * tiles; ++j2) {
        const int j = j2 >> 1, half = j2 & 1, at = done + j, left = u.n - (u.t0 + j) * kMaTile - 64 * half;
        // the waits' verdict is a warp's: tensor memory is read by whole warps
        ok = __all_sync(0xffffffffu, wait(&B.s_full[w][half], at));
        if (!ok) break;
        tc_fence_after();
        const uint32_t s_half = s_tm + (uint32_t)half * 64u;
        float v[64];
        tmem_ld32(s_half, v);
        tmem_ld32(s_half + 32u, v + 32);
        tmem_wait_ld();
        if (left < 64) {
#pragma unroll
          for (int x = 0; x < 64; ++x)
            if (x >= left) v[x] = -INFINITY;
        }
        float m[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
        for (int x = 4; x + 8 <= 64; x += 8)
#pragma unroll
          for (int z = 0; z < 4; ++z) m[z] = fmax3(m[z], v[x + 2 * z], v[x + 2 * z + 1]);
        m[0] = fmax3(m[0], v[60], v[61]);
        m[1] = fmax3(m[1], v[62], v[63]);
        const float mx = fmaxf(fmax3(m[0], m[1], m[2]), m[3]) * f;      // (the factor is positive)
        if (__any_sync(0xffffffffu, mx > ref + kMaSlack)) {
          float down = 1.f;
          if (mx > ref + kMaSlack) {
            down = ex2_approx(ref - mx);                // ref = -inf gives 0
            ref = mx;
          }
          l *= down;
          if (j2 > 0) {                                 // the products of the half before may still be adding to O
            ok = __all_sync(0xffffffffu, wait(&B.pv_done[w][half ^ 1], half ? at : at - 1));
            if (!ok) break;
            tc_fence_after();
#pragma unroll 1
            for (int x = 0; x < kD; x += 16) {
              float o[16];
              tmem_ld16(o_tm + x, o);
              tmem_wait_ld();
              uint32_t y[16];
#pragma unroll
              for (int z = 0; z < 16; ++z) y[z] = __float_as_uint(o[z] * down);
              tmem_st16(o_tm + x, y);
            }
          }
        }
        // The tiles' warpgroups take turns at the exponentials: while one is at them, the other loads and looks for the maximum.
        if (u.two && (w == 1 || u.done2 + j2 > 0)) ok = __all_sync(0xffffffffu, wait(&B.turn[w], 2 * u.done2 + j2 - (w == 0)));
        if (!ok) {
          tmem_wait_st();                               // (O may have been scaled: nothing is on its way when the CTA gives up its tensor memory)
          break;
        }
        const float m_use = ref == -INFINITY ? 0.f : ref;               // only logits of -inf so far: they weigh nothing
        const f32x2 ff = f2_make(f, f), minus_m = f2_make(-m_use, -m_use);
        f32x2 sum0 = f2_make(0.f, 0.f), sum1 = sum0;
#pragma unroll
        for (int x = 0; x < 64; x += 32) {
          uint32_t p[16];
#pragma unroll
          for (int y = 0; y < 32; y += 4) {
            const f32x2 a0 = f2_fma(f2_make(v[x + y], v[x + y + 1]), ff, minus_m), a1 = f2_fma(f2_make(v[x + y + 2], v[x + y + 3]), ff, minus_m);
            const float e0 = ex2_approx(f2_lo(a0)), e1 = ex2_approx(f2_hi(a0)), e2 = ex2_approx(f2_lo(a1)), e3 = ex2_approx(f2_hi(a1));
            sum0 = f2_add(sum0, f2_make(e0, e1));
            sum1 = f2_add(sum1, f2_make(e2, e3));
            p[y / 2] = pack_bf16x2(e0, e1);
            p[y / 2 + 1] = pack_bf16x2(e2, e3);
          }
          tmem_st16(s_half + x / 2, p);                 // P where S has been read already
          if (x == 0 && u.two) warp_arrive(&B.turn[1 - w]);
        }
        tmem_wait_st();
        tc_fence_before();
        warp_arrive(&B.p_full[w][half]);
        sum0 = f2_add(sum0, sum1);
        l += f2_lo(sum0) + f2_hi(sum0);
      }
      // ---- the row's result ----
      if (ok && tiles > 0) ok = __all_sync(0xffffffffu, wait(&B.pv_done[w][1], done + tiles - 1));
      if (ok) {
        tc_fence_after();
        const bool whole = u.whole, some = l != 0.f && live;   // (as cross_some)
        float* const part = a.part + (long long)(2 * blockIdx.x + (u.t0 == 0)) * kMaRows * (kD + 2);
        const long long row = cross_out_row(c, mine, u.h);
        __nv_bfloat16* const out = reinterpret_cast<__nv_bfloat16*>(c.out);
        constexpr int kChunks = kD / 8;
        if (!whole) {
          // four dims of all 256 rows after the other: a thread's stores lie beside those of the next row's
          float4* const to = reinterpret_cast<float4*>(part) + w * 128 + r;
#pragma unroll
          for (int x = 0; x < kD / 32; ++x) {
            if (tiles <= 0) break;                      // (none of its rows is there)
            float o[32];
            tmem_ld32(o_tm + x * 32, o);
            tmem_wait_ld();
#pragma unroll
            for (int y = 0; y < 32; y += 4) to[(32 * x + y) / 4 * kMaRows] = make_float4(o[y], o[y + 1], o[y + 2], o[y + 3]);
          }
        } else {
          // By way of the warp's rows of Q's tile, which no product reads any more, for stores of whole rows.  16-byte chunk k of row r is at k ^ r.
          const uint32_t staged = q_at + (uint32_t)w * C::kTileBytesD + (uint32_t)(warp & 3) * (32u * 2u * kD);
          const uint32_t to_row = staged + (uint32_t)lane * (2u * kD);
          const float norm = some ? 1.f / l : 0.f;
          if (tiles > 0) {
#pragma unroll
            for (int x = 0; x < kD / 32; ++x) {
              float o[32];
              tmem_ld32(o_tm + x * 32, o);
              tmem_wait_ld();
#pragma unroll
              for (int y = 0; y < 32; ++y) o[y] = some ? o[y] * norm : 0.f;
#pragma unroll
              for (int y = 0; y < 32; y += 8)
                many_sts128(to_row + (uint32_t)((((32 * x + y) / 8) ^ (lane & (kChunks - 1))) * 16), pack_bf16x2(o[y], o[y + 1]), pack_bf16x2(o[y + 2], o[y + 3]),
                            pack_bf16x2(o[y + 4], o[y + 5]), pack_bf16x2(o[y + 6], o[y + 7]));
            }
          }
          __syncwarp();
          const int k = lane % kChunks, in_tile = w * 128 + (warp & 3) * 32;
#pragma unroll 8
          for (int z = 0; z < 32; z += 32 / kChunks) {
            const int at = z + lane / kChunks;
            const long long to = __shfl_sync(0xffffffffu, row, at);
            if (u.rho0 + in_tile + at >= R) continue;
            reinterpret_cast<uint4*>(out + to * kD)[k] = tiles > 0 ? lds128(staged + (uint32_t)at * (2u * kD) + (uint32_t)((k ^ (at & (kChunks - 1))) * 16)) : make_uint4(0u, 0u, 0u, 0u);
          }
        }
        if (rho < R) {
          if (whole) {
            if (c.lse) c.lse[row] = some ? fmaf(ref, 0.6931471805599453f, logf(l)) : -INFINITY;
          } else {
            reinterpret_cast<float2*>(part + kMaRows * kD)[w * 128 + r] = make_float2(ref, l);
          }
        }
        tc_fence_before();
      }
      warp_arrive(&B.q_free[w]);
      return ok;
    });
  }
  __syncthreads();
  if (warp == kMaSoftmax + 1) tmem_dealloc(tmem, 512);
}

int many_ctas(int sm_count) { return sm_count < kMaxCtas ? sm_count : kMaxCtas; }

}  // namespace

template <int kD> cudaError_t many_init() {
  cudaFuncAttributes has;
  const cudaError_t e = cudaFuncGetAttributes(&has, cross_many_kernel<kD>);
  if (e != cudaSuccess) return e;
  if (has.numRegs != kMaRegs) return cudaErrorInvalidDeviceFunction;   // its warpgroups would wait for registers that are not there
  return cudaFuncSetAttribute(cross_many_kernel<kD>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)ManyConfig<kD>::kSmem);
}
cudaError_t cross_many_init() {
  const cudaError_t e = many_init<64>();
  return e != cudaSuccess ? e : many_init<128>();
}

bool cross_many_shape(const CrossProblem& c) { return (c.d == 64 || c.d == 128) && c.rows() >= kManyRows; }

bool cross_many_supported(const CrossProblem& c) {
  if (!cross_many_shape(c) || !cross_map_fits(c, c.K) || !cross_map_fits(c, c.V)) return false;
  const long long units = (long long)c.sources * c.Hkv * ((c.rows() + kMaRows - 1) / kMaRows);
  return ((long long)c.n_rows / kMaTile + 1 + kMaAhead) * units <= 0x7FFFFFFFll;   // tiles are counted in 32 bits
}

// About how long a call takes: 6 us, and 2.95 (head_dim 64: 1.9) per tile of a CTA, of which it has four at least or all of a unit's, and two for ends and
// beginnings of units.  Measured, 8 sources x 8 KV heads of 128, 128 query rows: 500 rows 17 us, 4000 rows 54 (in passes of 32 rows 66 and 145); one
// source: 4000 rows 21, 30000 46 (20 and 100); 4 sources of 100 rows, 80 query rows 12.3 (20).
double cross_many_us(const CrossProblem& c, int sm_count) {
  const double units = (double)c.sources * c.Hkv * (double)((c.rows() + kMaRows - 1) / kMaRows), of_unit = (double)((c.n_rows + kMaTile - 1) / kMaTile);
  const double tiles = units * of_unit / sm_count + 2.0, least = of_unit < 2.0 ? 3.0 : 4.0;
  return 6.0 + (c.d == 64 ? 1.9 : 2.95) * (tiles > least ? tiles : least);
}

size_t cross_many_bytes(const CrossProblem& c, int sm_count) {
  if (!cross_many_shape(c)) return 0;
  return (size_t)many_ctas(sm_count) * (2 * kMaRows * (c.d + 2) * sizeof(float) + sizeof(int2));
}

cudaError_t launch_cross_many(void* state, const CrossProblem& c, float* part, int sm_count, long long wait_limit, unsigned int* dev_status, cudaStream_t st) {
  CUtensorMap tmK, tmV;
  if (!make_cross_map((TcState*)state, &tmK, c, c.K, kMaTile) || !make_cross_map((TcState*)state, &tmV, c, c.V, kMaTile)) return cudaErrorInvalidValue;
  const int ctas = many_ctas(sm_count);
  CrossManyArgs a{};
  a.c = c; a.part = part; a.dev_status = dev_status; a.wait_limit = wait_limit;
  a.row_tiles = (int)((c.rows() + kMaRows - 1) / kMaRows);
  a.begins = reinterpret_cast<int2*>(part + (size_t)2 * ctas * kMaRows * (c.d + 2));
  const cudaError_t e = c.d == 64 ? launch_chained(cross_many_kernel<64>, dim3((unsigned int)ctas), kMaThreads, ManyConfig<64>::kSmem, st, tmK, tmV, a)
                                  : launch_chained(cross_many_kernel<128>, dim3((unsigned int)ctas), kMaThreads, ManyConfig<128>::kSmem, st, tmK, tmV, a);
  if (e != cudaSuccess) return e;
  return c.d == 64 ? launch_merge<64, kMaRows>(c, part, a.begins, a.row_tiles, ctas, st) : launch_merge<128, kMaRows>(c, part, a.begins, a.row_tiles, ctas, st);
}

}  // namespace restkv
