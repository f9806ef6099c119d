// What the tensor-core kernels of the paged attention share: their arguments, the work dealt out over CTAs, a row's result.
#pragma once

#include "paged.cuh"
#include "tc_common.cuh"

namespace restkv {
namespace {

constexpr int kMaxCtas = 512;

struct PagedMmaArgs {
  PagedCache c;
  RowsView Q;
  __nv_bfloat16* out;
  float* lse;        // or null
  float* part;       // per CTA two of: o [rows, d], (m, l) [rows]; without clusters
  int4* begins;      // per CTA, chunks: unit and tile of it that it begins with; whether pages were bad in units that it begins, in one that it goes on with
  int row_tiles;     // units per KV head
  int cluster;       // CTAs per unit, 0: tiles of all units end to end
  long long wait_limit;
};

// A capped logit is cap * tanh(t), t = s / cap.  For |t| <= 0.6 an odd polynomial (minimax, relative error 9.3e-8, 1.8e-7 with the fp32
// rounding of the chain), past it 1 - 2 / (1 + e^2t) with two trips to the special-function unit (2^-22, less than 2^-21 of tanh(0.6)).  That
// one alone would be off by 2^-22 of the cap for a small logit under a large cap.
constexpr float kTanhNear = 0.6f;
__device__ __forceinline__ f32x2 tanh_near(f32x2 t) {
  const f32x2 z = f2_mul(t, t);
  f32x2 p = f2_make(0.0154755134f, 0.0154755134f);
  p = f2_fma(p, z, f2_make(-0.0521015525f, -0.0521015525f));
  p = f2_fma(p, z, f2_make(0.133101761f, 0.133101761f));
  p = f2_fma(p, z, f2_make(-0.333323091f, -0.333323091f));
  p = f2_fma(p, z, f2_make(0.99999994f, 0.99999994f));
  return f2_mul(p, t);
}
__device__ __forceinline__ float tanh_far(float t) { return fmaf(-2.f, rcp_approx(1.f + ex2_approx(t * 2.f * kLog2e)), 1.f); }
__device__ __forceinline__ void tanh_any(float& t0, float& t1) {
  const f32x2 near = tanh_near(f2_make(t0, t1));
  const float far0 = tanh_far(t0), far1 = tanh_far(t1);
  t0 = fabsf(t0) <= kTanhNear ? f2_lo(near) : far0;
  t1 = fabsf(t1) <= kTanhNear ? f2_hi(near) : far1;
}

__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ float lower(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float upper(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// Tiles dealt out end to end: CTA x of `ctas` has those from boundary x to boundary x + 1.  A boundary is start(x) = all * x / ctas, but
// moved to the near end of its unit where that is at most `snap` tiles away: a CTA that ends one unit and begins another pays for
// prologue and merge twice, in which it would go through as many tiles.
struct Deal {
  int ctas, each, more, snap;
  __device__ __forceinline__ Deal(int all, int grid, int most) : ctas(all < grid ? all : grid), each(all / ctas), more(all - each * ctas) {
    snap = (each - 1) / 2 < most ? (each - 1) / 2 : most;   // less than half a share: no share vanishes
  }
  __device__ __forceinline__ int start(int x) const { return x * each + x * more / ctas; }
  // tile `at` of a unit of `tiles`: where a boundary there goes, as tile of the unit
  __device__ __forceinline__ int moved(int at, int tiles) const {
    const int left = tiles - at;
    return at <= snap && at <= left ? 0 : left <= snap ? tiles : at;
  }
  // the last CTA whose start is not past `tile`
  __device__ __forceinline__ int last(int tile) const {
    int x = (int)((float)tile / ((float)each + (float)more / (float)ctas));
    x = x < ctas ? x : ctas - 1;
    while (x > 0 && start(x) > tile) --x;
    while (x + 1 < ctas && start(x + 1) <= tile) ++x;
    return x;
  }
  // the CTAs that have tiles of the unit [u0, u0 + tiles): the first of them its beginning
  __device__ __forceinline__ int first_of(int u0, int tiles) const { return last(u0 + (snap < tiles / 2 ? snap : tiles / 2)); }
  __device__ __forceinline__ int last_of(int u0, int tiles) const {
    return last(u0 + tiles - 1 - (snap < (tiles - 1) / 2 ? snap : (tiles - 1) / 2));
  }
};

// Entries of the kernel for few tokens: sequences, or with lengths per head the KV heads of all sequences; each has units of as many tiles.
__device__ __forceinline__ int entries_of(const PagedCache& c) { return c.per_head ? c.batch * c.Hkv : c.batch; }
__device__ __forceinline__ int units_of(const PagedCache& c, int row_tiles) { return c.per_head ? row_tiles : c.Hkv * row_tiles; }
__device__ __forceinline__ int entry_tiles(const PagedCache& c, int e, int tile_rows) {
  const int n = c.per_head ? paged_length(c, e / c.Hkv, e % c.Hkv) : paged_length(c, e, 0);
  const int t = (n + tile_rows - 1) / tile_rows;
  return t > 0 ? t : 1;     // a unit without rows has its outputs written, too
}

// By a whole warp: a CTA's run of tiles [tile, end), the entry that `tile` lies in, the entry's first tile and tiles per unit.
struct Run {
  int tile, end, entry, first, tiles;
};
__device__ __forceinline__ Run find_run(const PagedCache& c, int row_tiles, int tile_rows, int most, int x, int grid) {
  const int lane = threadIdx.x & 31;
  const int entries = entries_of(c), units = units_of(c, row_tiles);
  const int t0 = lane < entries ? entry_tiles(c, lane, tile_rows) : 0;
  int sum = t0 * units;
  for (int e = 32 + lane; e < entries; e += 32) sum += entry_tiles(c, e, tile_rows) * units;
  const int all = __reduce_add_sync(0xffffffffu, sum);
  const Deal deal(all, grid, most);
  Run r{0, 0, 0, 0, 1};
  if (x >= deal.ctas) return r;
  r.tile = r.end = all;
  int want = deal.start(x), before = 0;
  bool have = false;
  for (int base = 0; base < entries; base += 32) {
    const int t = base == 0 ? t0 : base + lane < entries ? entry_tiles(c, base + lane, tile_rows) : 0;
    int upto = t * units;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const int o = __shfl_up_sync(0xffffffffu, upto, off);
      if (lane >= off) upto += o;
    }
    for (;;) {             // both boundaries of the CTA may lie in these entries
      const unsigned int past = __ballot_sync(0xffffffffu, before + upto > want);
      if (!past) break;
      const int at = __ffs((int)past) - 1;
      const int tiles = __shfl_sync(0xffffffffu, t, at), first = before + __shfl_sync(0xffffffffu, upto, at) - tiles * units;
      const int unit0 = first + (want - first) / tiles * tiles, boundary = unit0 + deal.moved(want - unit0, tiles);
      if (!have) {
        have = true;
        r = Run{boundary, all, base + at, first, tiles};
        if (x + 1 == deal.ctas) return r;
        want = deal.start(x + 1);
      } else {
        r.end = boundary;
        return r;
      }
    }
    before += __shfl_sync(0xffffffffu, upto, 31);
  }
  return r;
}

// Dims kPer v .. of a query row's result.
template <int kD, int kPer>
__device__ __forceinline__ void write_row(const PagedMmaArgs& a, int b, int h, int rho, int count, int v, const float (&acc)[kPer], float mm, float ll) {
  const PagedCache& c = a.c;
  const int i = rho / c.G, g = rho - i * c.G;
  const bool some = ll > 0.f && i < count;
  const long long at = ((long long)b * c.Hq + h * c.G + g) * c.n_tokens + i;
  const float f = some ? 1.f / ll : 0.f;
  uint32_t w[kPer / 2];
#pragma unroll
  for (int x = 0; x < kPer / 2; ++x) w[x] = some ? pack_bf16x2(acc[2 * x] * f, acc[2 * x + 1] * f) : 0u;
  __nv_bfloat16* const to = a.out + at * kD + kPer * v;
  if constexpr (kPer == 4) *reinterpret_cast<uint2*>(to) = make_uint2(w[0], w[1]);
  else *reinterpret_cast<uint32_t*>(to) = w[0];
  if (v == 0 && a.lse) a.lse[at] = some ? fmaf(mm, 0.6931471805599453f, logf(ll)) : -INFINITY;
}
template <int kD>
__device__ __forceinline__ void write_row(const PagedMmaArgs& a, int b, int h, int rho, int count, int v, float4 acc, float mm, float ll) {
  const float x[4] = {acc.x, acc.y, acc.z, acc.w};
  write_row<kD, 4>(a, b, h, rho, count, v, x, mm, ll);
}
__device__ __forceinline__ void fma4(float4& acc, float4 x, float f) {
  acc.x = fmaf(x.x, f, acc.x); acc.y = fmaf(x.y, f, acc.y); acc.z = fmaf(x.z, f, acc.z); acc.w = fmaf(x.w, f, acc.w);
}

// What a CTA works on without clusters, in shared memory: it is needed before the tiles and after them, and registers are short between.
struct Piece {
  Run run;
  int unit, t0, t1;        // tiles [t0, t1) of the unit
  int whole;               // no other CTA has tiles of it
  template <class TilesOf> __device__ __forceinline__ void cut(int units, TilesOf&& tiles_of) {   // at run.tile
    if (run.tile >= run.first + run.tiles * units) {     // the next entry
      run.first += run.tiles * units;
      run.tiles = tiles_of(++run.entry);
    }
    const int k = (run.tile - run.first) / run.tiles, begin = run.first + k * run.tiles;
    unit = run.entry * units + k;
    t0 = run.tile - begin;
    t1 = run.end - begin < run.tiles ? run.end - begin : run.tiles;
    whole = t0 == 0 && t1 == run.tiles;
  }
};

}  // namespace
}  // namespace restkv
