// The best continuations of a request's hypotheses: scores[k] + logits[k,v] - log sum exp(logits[k,:]), over hypotheses and tokens.
//
// One pass over the logits.  A block goes through a slice of a row: its maximum and sum of exponentials, and its n_out largest logits.  A second kernel
// joins a request's slices: normalisers, scores in 64 bits, the n_out best.
// Largest of a block: groups of four threads name their largest logit; the n_out-th of those bounds the n_out-th of the slice from below, and what
// reaches it, a few more than n_out as a rule, is read once more (by the threads whose batch of pieces has some), collected in shared memory and
// ranked by counting.  Where that is more than the list holds (a slice of equal logits, say) the bound is found anew among logits with their tokens,
// of which no two are equal, and where that does not do either the largest are taken one by one.  The second kernel does the same with scores.
// Logits of -inf are no candidates in either; requests that run out of others look for them in the rows at the end.
// What bounds it: no one unit for large calls; bytes, and an exponential per logit (16 per clock and SM: 14 us for the 67 million logits of 512 rows of
// 131072 whose bytes take 21), are worked off by turns in each block, and where the blocks are more than one wave the last is not full (1024 of 740 places there).  For
// small calls two launches, each a chain of loads and a few barriers.  Where more candidates of a request reach the bound than the second kernel's list holds,
// they are taken one by one: 64 wanted of 64 hypotheses of 32000 tokens take 102 to 110 us with scores within 2 of one another, 2.4 ms within 10.
#include <math.h>

#include "beam.cuh"
#include "row_pieces.cuh"
#include "sm100_ptx.cuh"

namespace restkv {

namespace {

using namespace ptx;

constexpr int kBeThreads = 256, kBeWarps = kBeThreads / 32, kBePerSm = 5;
constexpr int kGroups = kBeThreads / 4;         // at least kBeamOut
constexpr int kList = 2048, kJoinList = 512;
constexpr float kLog2e = 1.4426950408889634f;
static_assert((kGroups & (kGroups - 1)) == 0, "places turn round");
static_assert(kGroups >= kBeamOut, "a threshold needs as many groups as continuations");

typedef unsigned long long u64;

// A logit and its token as one key: larger logits first, then lower tokens.  0 is no candidate.
__device__ __forceinline__ u64 make_key(float x, int token) { return (u64)float_key(x + 0.f) << 32 | (unsigned int)~token; }   // (-0 is 0)
__device__ __forceinline__ float key_logit(u64 key) {
  const unsigned int k = (unsigned int)(key >> 32);
  return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k);
}
__device__ __forceinline__ int key_token(u64 key) { return (int)~(unsigned int)key; }

__device__ __forceinline__ float usable(float x) { return fminf(fmaxf(x, -INFINITY), 3.402823466e38f); }   // NaN: -inf; +inf: the largest number

// What a row's hypothesis asks for: its logits (0), its one continuation (1), nothing that is above -inf (2).
__device__ __forceinline__ int row_kind(const BeamProblem& p, int row) {
  if (!(p.scores[row] > -INFINITY)) return 2;
  return p.finished && p.finished[row] ? 1 : 0;
}

// The n-th largest of the groups' values; ends with a barrier.  A group ranks its own value, a quarter of the others per thread.
template <typename K> __device__ __forceinline__ K nth_of_groups(K mine, int n, K (&group_s)[kGroups], K& limit_s) {
  const int t = threadIdx.x, group = t >> 2;
#pragma unroll
  for (int x = 1; x <= 2; x <<= 1) {
    const K o = __shfl_xor_sync(0xffffffffu, mine, x);
    mine = o > mine ? o : mine;
  }
  if ((t & 3) == 0) group_s[group] = mine;
  __syncthreads();
  int before = 0;
#pragma unroll
  for (int i = 0; i < kGroups / 4; ++i) {
    const int g = 4 * i + (t & 3);
    const K o = group_s[g];
    before += o > mine || (o == mine && g < group);
  }
  before += __shfl_xor_sync(0xffffffffu, before, 1);
  before += __shfl_xor_sync(0xffffffffu, before, 2);
  if (before == n - 1 && (t & 3) == 0) limit_s = mine;
  __syncthreads();
  return limit_s;
}

// How many of `count` come before each of them, four threads to one.
template <class Before, class Use> __device__ __forceinline__ void rank(int count, Before&& comes_before, Use&& use) {
  for (int x0 = 0; x0 < count; x0 += kBeThreads / 4) {
    const int x = x0 + ((int)threadIdx.x >> 2);
    int before = 0;
    if (x < count) {
#pragma unroll 4
      for (int y = threadIdx.x & 3; y < count; y += 4) before += comes_before(x, y);
    }
    before += __shfl_xor_sync(0xffffffffu, before, 1);
    before += __shfl_xor_sync(0xffffffffu, before, 2);
    if (x < count && (threadIdx.x & 3) == 0) use(x, before);
  }
}

template <typename T> struct Vec;      // 16 bytes of logits
template <> struct Vec<float> {
  static constexpr int kPer = 4;
  uint4 u;
  __device__ float at(int i) const { return __uint_as_float((&u.x)[i]); }
  __device__ void set(int i, float x) { (&u.x)[i] = __float_as_uint(x); }
};
template <> struct Vec<__nv_bfloat16> {
  static constexpr int kPer = 8;
  uint4 u;
  __device__ float at(int i) const {
    const unsigned int w = (&u.x)[i >> 1];
    return __uint_as_float(i & 1 ? w & 0xFFFF0000u : w << 16);
  }
  __device__ void set(int i, float x) {       // (a bf16 value)
    unsigned int& w = (&u.x)[i >> 1];
    const unsigned int b = __float_as_uint(x) >> 16;
    w = i & 1 ? (w & 0xFFFFu) | b << 16 : (w & 0xFFFF0000u) | b;
  }
};

// 16 of the 32 bytes of two pieces, from byte `off` on (even).
__device__ __forceinline__ uint4 shifted(uint4 a, uint4 b, unsigned int off) {
  unsigned int w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  if (off & 8) {
#pragma unroll
    for (int i = 0; i < 6; ++i) w[i] = w[i + 2];
  }
  if (off & 4) {
#pragma unroll
    for (int i = 0; i < 5; ++i) w[i] = w[i + 1];
  }
  if (off & 2) {
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], 16);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}

struct __align__(8) SliceStats { float top, sum; };   // of a slice: its maximum and the sum of exp(x - top); no finite logit: -inf, 0

// grid: rows x slices, slices running fastest.  A slice is kBatches batches of kBatch * kBeThreads pieces of 16 bytes of a row.
// kRagged: the rows end inside a piece, behind which is nobody's memory.  (A kernel of its own, for the others have no register to spare.  The ends of
// rows token by token take longer: 255 rows of 50257 of 16 bits 17.2 us, 256, which end with a piece, 16.6; 512 of 131072 as before, 35.8.)
template <typename T, int kBatch, int kBatches, bool kRagged>
__global__ void __launch_bounds__(kBeThreads, kBePerSm) beam_slice_kernel(const BeamProblem p, int slices, SliceStats* __restrict__ stats, u64* __restrict__ lists) {
  using V = Vec<T>;
  constexpr int kPer = V::kPer, kMine = kBatch * kPer;      // logits of a thread in a batch
  __shared__ __align__(16) float group_s[kGroups];
  __shared__ u64 group_key_s[kGroups], limit_key_s;
  __shared__ float limit_s, top_s[kBeWarps], sum_s[kBeWarps];
  __shared__ int count_s, anew_s, hits_s;   // of the list, of the list as it is found anew: no counter is set back, for a warp may be late to read it
  __shared__ unsigned short hit_s[kBatches * kBeThreads];
  __shared__ u64 list_s[kList], best_s[kBeWarps];
  const int row = blockIdx.x / slices, slice = blockIdx.x - row * slices, t = threadIdx.x, lane = t & 31, warp = t >> 5;
  grid_dependency_wait();
  grid_dependency_launch();
  if (row_kind(p, row) != 0) return;
  const T* const from = reinterpret_cast<const T*>(p.logits) + row * p.stride;
  // A thread's tokens do not depend on where in its 16-byte pieces the row begins: equal rows have equal sums, bit for bit.
  const unsigned int off = (unsigned int)(reinterpret_cast<uintptr_t>(from) & 15u);   // bytes of the row before in the row's first piece
  const uint4* const pieces = reinterpret_cast<const uint4*>(reinterpret_cast<uintptr_t>(from) & ~(uintptr_t)15);
  const RowPieces<kRagged> in_row(off, p.vocab, (int)sizeof(T));
  const int piece0 = slice * (kBatches * kBatch * kBeThreads) + t;
  auto piece_of = [&](int b, int y) { return piece0 + (b * kBatch + y) * kBeThreads; };
  auto token_of = [&](int b, int e) { return piece_of(b, e / kPer) * kPer + e % kPer; };     // of the thread's e-th logit of batch b
  if (t == 0) count_s = anew_s = hits_s = 0;
  float top = -INFINITY, sum = 0.f, most[kBatches];         // of the thread, and of its batches
#pragma unroll
  for (int b = 0; b < kBatches; ++b) {
    V v[kBatch];
#pragma unroll
    for (int y = 0; y < kBatch; ++y) v[y].u = piece_of(b, y) < in_row.loaded ? __ldcs(pieces + piece_of(b, y)) : make_uint4(0u, 0u, 0u, 0u);
    if (off) {
#pragma unroll
      for (int y = 0; y < kBatch; ++y) {
        uint4 next = make_uint4(__shfl_down_sync(0xffffffffu, v[y].u.x, 1), __shfl_down_sync(0xffffffffu, v[y].u.y, 1), __shfl_down_sync(0xffffffffu, v[y].u.z, 1),
                                __shfl_down_sync(0xffffffffu, v[y].u.w, 1));
        if (lane == 31) next = piece_of(b, y) + 1 < in_row.loaded ? __ldg(pieces + piece_of(b, y) + 1) : make_uint4(0u, 0u, 0u, 0u);
        v[y].u = shifted(v[y].u, next, off);
      }
    }
    if (!kRagged || (slice + 1) * (kBatches * kBatch * kBeThreads) > in_row.inside) {
#pragma unroll
      for (int y = 0; y < kBatch; ++y) {
        if (kRagged ? piece_of(b, y) < in_row.inside : token_of(b, y * kPer + kPer - 1) < p.vocab) continue;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          const int token = token_of(b, y * kPer + i);
          if (token >= p.vocab) v[y].set(i, -INFINITY);
          else if (kRagged) v[y].set(i, to_f32<T>(from[token]));
        }
      }
    }
    float m0 = -INFINITY, m1 = -INFINITY;                   // (a NaN is passed over)
#pragma unroll
    for (int e = 0; e < kMine; e += 4) {
      m0 = fmax3(m0, v[e / kPer].at(e % kPer), v[e / kPer].at(e % kPer + 1));
      m1 = fmax3(m1, v[e / kPer].at(e % kPer + 2), v[e / kPer].at(e % kPer + 3));
    }
    most[b] = fmaxf(m0, m1);
    const float next = fmaxf(top, most[b]), of = next == -INFINITY ? 0.f : next;
    sum *= ex2_approx((top - of) * kLog2e);
    top = next;
    f32x2 s0 = f2_make(0.f, 0.f), s1 = s0;
    const f32x2 minus = f2_make(-of, -of), scale = f2_make(kLog2e, kLog2e);
#pragma unroll
    for (int e = 0; e < kMine; e += 4) {
      const V& w = v[e / kPer];
      const int i = e % kPer;
      // the difference first: large terms have small ones, whose rounding is small
      const f32x2 x = f2_mul(f2_add(f2_make(w.at(i), w.at(i + 1)), minus), scale), y = f2_mul(f2_add(f2_make(w.at(i + 2), w.at(i + 3)), minus), scale);
      s0 = f2_add(s0, f2_make(ex2_approx(f2_lo(x)), ex2_approx(f2_hi(x))));
      s1 = f2_add(s1, f2_make(ex2_approx(f2_lo(y)), ex2_approx(f2_hi(y))));
    }
    s0 = f2_add(s0, s1);
    sum += f2_lo(s0) + f2_hi(s0);
  }
  // the thread's e-th logit of batch b once more, as it counts
  auto again = [&](int b, int e) {
    const int token = token_of(b, e);
    return token < p.vocab ? usable(to_f32<T>(from[token])) : -INFINITY;
  };
  if (!(sum < INFINITY)) {   // a NaN or +inf among the logits shows in the sum: all anew of what counts in their place
    top = -INFINITY;
#pragma unroll
    for (int b = 0; b < kBatches; ++b) {
      most[b] = -INFINITY;
#pragma unroll 1
      for (int e = 0; e < kMine; ++e) most[b] = fmaxf(most[b], again(b, e));
      top = fmaxf(top, most[b]);
    }
    sum = 0.f;
#pragma unroll 1
    for (int e = 0; e < kBatches * kMine; ++e) sum += top == -INFINITY ? 0.f : ex2_approx((again(e / kMine, e % kMine) - top) * kLog2e);
  }
  const float limit = nth_of_groups(top, p.n_out, group_s, limit_s);
  // ---- the slice's statistics ----
  {
    float m = top;
#pragma unroll
    for (int x = 16; x > 0; x >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
    float s = m == -INFINITY ? 0.f : sum * ex2_approx((top - m) * kLog2e);
#pragma unroll
    for (int x = 16; x > 0; x >>= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
    if (lane == 0) { top_s[warp] = m; sum_s[warp] = s; }
  }
  // ---- what reaches the limit: the batches that have some are read once more, by all threads side by side ----
  if (top >= limit && top > -INFINITY) {
#pragma unroll
    for (int b = 0; b < kBatches; ++b)
      if (most[b] >= limit) hit_s[atomicAdd(&hits_s, 1)] = (unsigned short)(b * kBeThreads + t);
  }
  __syncthreads();
  constexpr int kAhead = 4;
  for (int x0 = t, all = hits_s * kMine; x0 < all; x0 += kAhead * kBeThreads) {
    float z[kAhead];
    int token[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int x = x0 + i * kBeThreads, hit = x < all ? hit_s[x / kMine] : 0, e = x % kMine;
      token[i] = token_of(hit / kBeThreads, e) + (hit % kBeThreads - t) * kPer;
      z[i] = x < all && token[i] < p.vocab ? to_f32<T>(from[token[i]]) : -INFINITY;
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      z[i] = usable(z[i]);
      if (!(z[i] >= limit) || z[i] == -INFINITY) continue;
      const int at = atomicAdd(&count_s, 1);
      if (at < kList) list_s[at] = make_key(z[i], token[i]);
    }
  }
  __syncthreads();
  int count = count_s;
  if (count > kList) {
    // too many of one size: a limit among logits with their tokens
    u64 best = 0;
#pragma unroll 1
    for (int e = 0; e < kBatches * kMine; ++e) {
      const float x = again(e / kMine, e % kMine);
      const u64 key = x > -INFINITY ? make_key(x, token_of(e / kMine, e % kMine)) : 0;
      best = key > best ? key : best;
    }
    const u64 limit_key = nth_of_groups(best, p.n_out, group_key_s, limit_key_s);
    if (best >= limit_key && best > 0) {
#pragma unroll 1
      for (int e = 0; e < kBatches * kMine; ++e) {
        const float x = again(e / kMine, e % kMine);
        const u64 key = x > -INFINITY ? make_key(x, token_of(e / kMine, e % kMine)) : 0;
        if (key >= limit_key && key > 0) {
          const int at = atomicAdd(&anew_s, 1);
          if (at < kList) list_s[at] = key;
        }
      }
    }
    __syncthreads();
    count = anew_s;
  }
  // a request's lists side by side: place k of all of them, then place k + 1
  const int request = row / p.beams, side = p.beams * slices;
  u64* const list = lists + (long long)request * side * p.n_out + ((int)blockIdx.x - request * side);
  if (count <= kList) {
    rank(count, [&](int x, int y) { return list_s[y] > list_s[x]; }, [&](int x, int before) {
      if (before < p.n_out) list[before * side] = list_s[x];
    });
    for (int x = count + t; x < p.n_out; x += kBeThreads) list[x * side] = 0;
  } else {
    u64 last = ~0ull;
    for (int k = 0; k < p.n_out; ++k) {
      u64 best = 0;
#pragma unroll 1
      for (int e = 0; e < kBatches * kMine; ++e) {
        const float x = again(e / kMine, e % kMine);
        const u64 key = x > -INFINITY ? make_key(x, token_of(e / kMine, e % kMine)) : 0;
        if (key < last && key > best) best = key;
      }
#pragma unroll
      for (int x = 16; x > 0; x >>= 1) {
        const u64 o = __shfl_xor_sync(0xffffffffu, best, x);
        best = o > best ? o : best;
      }
      __syncthreads();
      if (lane == 0) best_s[warp] = best;
      __syncthreads();
      last = best_s[0];
#pragma unroll
      for (int w = 1; w < kBeWarps; ++w) last = best_s[w] > last ? best_s[w] : last;
      if (t == 0) list[k * side] = last;             // (more than kList candidates: never 0)
    }
  }
  if (t == 0) {
    float m = top_s[0], s = 0.f;
#pragma unroll
    for (int w = 1; w < kBeWarps; ++w) m = fmaxf(m, top_s[w]);
#pragma unroll
    for (int w = 0; w < kBeWarps; ++w) s += top_s[w] == -INFINITY ? 0.f : sum_s[w] * ex2_approx((top_s[w] - m) * kLog2e);
    stats[blockIdx.x] = SliceStats{m, s};
  }
}

// A continuation by its score, hypothesis and key.  Scores are compared by their bits in an order of integers.
struct Candidate {
  u64 score, key;
  int beam;
  // (without branches: lanes that take different ones of them cost 240 cycles a comparison)
  __device__ bool before(const Candidate& o) const { return (score > o.score) | ((score == o.score) & ((beam < o.beam) | ((beam == o.beam) & (key > o.key)))); }
};
__device__ __forceinline__ u64 score_bits(double x) {
  const long long u = __double_as_longlong(x + 0.0);      // (-0 is 0)
  return (u64)(u ^ (u >> 63 | (long long)(1ull << 63)));
}
__device__ __forceinline__ double score_of(u64 bits) { return __longlong_as_double((long long)(bits >> 63 ? bits ^ 1ull << 63 : ~bits)); }

// grid: requests
template <typename T>
__global__ void __launch_bounds__(kBeThreads, 4) beam_join_kernel(const BeamProblem p, int slices, const SliceStats* __restrict__ stats, const u64* __restrict__ lists) {
  __shared__ __align__(16) float group_s[kGroups];
  __shared__ float limit_s;
  __shared__ int count_s, kind_s[kBeamsPerRequest];
  __shared__ double total_s[kBeamsPerRequest];    // normalisers ...
  __shared__ float score_s[kBeamsPerRequest], near_s[kBeamsPerRequest];   // ... and rounded
  __shared__ Candidate list_s[kJoinList], best_s[kBeWarps];
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5, row0 = (int)blockIdx.x * p.beams, n_out = p.n_out;
  grid_dependency_wait();
  grid_dependency_launch();
  if (t == 0) count_s = 0;
  // Candidate x of the request: the firsts of all slices of all hypotheses, then the seconds ...; so the groups whose largest make the limit have the
  // same share of the firsts (by lists one after the other, the 64th of 64 groups had lasts of lists only: 2300 us for 64 of 64 hypotheses).
  // A thread holds kHeld of the first 256 kHeld, on their way before the normalisers are known.
  constexpr int kHeld = 8;
  const int side = p.beams * slices, all = side * n_out;
  // 64 in turn to the 64 groups, each time 16 groups on: the four of a group come from different slices wherever there are several
  const int place = (t & 3) * kGroups + (((t >> 2) + kGroups / 4 * (t & 3)) & (kGroups - 1));
  u64 held[kHeld];
  auto hold = [&](int base) {
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      const int x = base + i * kBeThreads + place;
      held[i] = x < all ? __ldcg(lists + (long long)blockIdx.x * all + x) : 0;
    }
  };
  hold(0);
  for (int k = warp; k < p.beams; k += kBeWarps) {
    const int row = row0 + k, kind = row_kind(p, row);
    double total = 0.0;
    float m = -INFINITY, tops[2], sums[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const SliceStats* const of = stats + (long long)row * slices + lane + 32 * i;
      const float2 z = lane + 32 * i < slices ? __ldcg(reinterpret_cast<const float2*>(of)) : make_float2(-INFINITY, 0.f);
      tops[i] = z.x;
      sums[i] = z.y;
    }
    if (kind == 0) {
      m = fmaxf(tops[0], tops[1]);
      for (int x = lane + 64; x < slices; x += 32) m = fmaxf(m, __ldcg(&stats[(long long)row * slices + x].top));
#pragma unroll
      for (int x = 16; x > 0; x >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
      auto part = [&](float top, float sum) { return top > -INFINITY ? (double)sum * (double)ex2_approx((top - m) * kLog2e) : 0.0; };
      double s = part(tops[0], sums[0]) + part(tops[1], sums[1]);
      for (int x = lane + 64; x < slices; x += 32) {
        const float2 z = __ldcg(reinterpret_cast<const float2*>(&stats[(long long)row * slices + x]));
        s += part(z.x, z.y);
      }
#pragma unroll
      for (int x = 16; x > 0; x >>= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
      total = (double)m + log(s);                 // (a row without candidates has none that would use it)
    }
    if (lane == 0) { kind_s[k] = kind; score_s[k] = p.scores[row]; total_s[k] = total; near_s[k] = (float)total; }
  }
  __syncthreads();
  // Scores in fp32 first, with bounds of what they are off by: the n_out-th largest lower bound bounds the n_out-th largest score, and what may
  // reach it is scored in 64 bits (an operation in 64 bits takes as long as a dozen others).
  struct Bounds {
    float least, most;
  };
  auto bounds = [&](int k, u64 key) {
    const float x = kind_s[k] == 0 ? key_logit(key) : 0.f, before = score_s[k], total = near_s[k];
    const float near = before + (x - total), off = 0x1p-21f * (fabsf(before) + fabsf(x) + fabsf(total));
    return Bounds{near - off, near + off};
  };
  auto key_at = [&](int k, int x, u64 key) {      // 0: no candidate
    const int kind = kind_s[k];
    return kind == 0 ? key : kind == 1 && x == k * slices ? make_key(0.f, p.pad_token) : 0;
  };
  auto candidate = [&](int k, u64 key) {
    return Candidate{score_bits(kind_s[k] == 0 ? (double)score_s[k] + ((double)key_logit(key) - total_s[k]) : (double)score_s[k]), key, k};
  };
  // a / b, b > 0, for which 1 / b is given: a below 2^21 by a product that is off by less than half of 1 / b
  auto quotient = [&](int a, int b, float inverse) { return all <= 1 << 21 ? (int)(((float)a + 0.5f) * inverse) : a / b; };
  const float per_side = 1.f / (float)side, per_slice = 1.f / (float)slices;
  auto some = [&](int base, auto&& use) {
#pragma unroll
    for (int i = 0; i < kHeld; ++i) {
      const int x = base + i * kBeThreads + place;
      if (x >= all) break;
      const int k = quotient(x - quotient(x, side, per_side) * side, slices, per_slice);
      const u64 own = key_at(k, x, held[i]);
      if (own) use(k, own);
    }
  };
  bool first = true;                              // what is held is where `each` begins
  auto each = [&](auto&& use) {
#pragma unroll 1
    for (int base = 0; base < all; base += kHeld * kBeThreads) {
      if (!first) hold(base);
      some(base, use);
      first = all <= kHeld * kBeThreads;
    }
  };
  float top = -INFINITY;
  each([&](int k, u64 key) { top = fmaxf(top, bounds(k, key).least); });      // (a NaN, of infinities, bounds nothing)
  const float limit = nth_of_groups(top, n_out, group_s, limit_s);
  each([&](int k, u64 key) {
    if (bounds(k, key).most < limit) return;
    const int at = atomicAdd(&count_s, 1);
    if (at < kJoinList) list_s[at] = candidate(k, key);
  });
  __syncthreads();
  const int count = count_s;
  auto put = [&](int at, const Candidate& c) {
    const long long to = (long long)blockIdx.x * n_out + at;
    p.parents[to] = c.beam;
    p.tokens[to] = key_token(c.key);
    p.scores_out[to] = (float)score_of(c.score);
  };
  if (count <= kJoinList) {
    rank(count, [&](int x, int y) { return list_s[y].before(list_s[x]); }, [&](int x, int before) {
      if (before < n_out) put(before, list_s[x]);
    });
  } else {
    Candidate last{~0ull, ~0ull, -1};
    for (int k = 0; k < n_out; ++k) {
      Candidate best{0, 0, 0};                    // key 0: none
      each([&](int k, u64 key) {
        const Candidate c = candidate(k, key);
        if (last.before(c) && (!best.key || c.before(best))) best = c;
      });
#pragma unroll
      for (int x = 16; x > 0; x >>= 1) {
        const Candidate o{__shfl_xor_sync(0xffffffffu, best.score, x), __shfl_xor_sync(0xffffffffu, best.key, x), __shfl_xor_sync(0xffffffffu, best.beam, x)};
        if (o.key && (!best.key || o.before(best))) best = o;
      }
      __syncthreads();
      if (lane == 0) best_s[warp] = best;
      __syncthreads();
      last = best_s[0];
#pragma unroll
      for (int w = 1; w < kBeWarps; ++w)
        if (best_s[w].key && (!last.key || best_s[w].before(last))) last = best_s[w];
      if (t == 0) put(k, last);
    }
  }
  if (count >= n_out || warp != 0) return;
  // Fewer continuations above -inf than are wanted: those of -inf, by hypothesis and token, as far as there are any.
  int have = count;
  for (int k = 0; k < p.beams && have < n_out; ++k) {
    const int row = row0 + k;
    const bool ended = p.finished && p.finished[row];
    if (kind_s[k] == 1) continue;                 // its one continuation is there already
    const T* const from = reinterpret_cast<const T*>(p.logits) + row * p.stride;
    const int tokens = ended ? 1 : p.vocab;
    for (int v0 = 0; v0 < tokens && have < n_out; v0 += 32) {
      const int v = v0 + lane;
      const bool is = v < tokens && (kind_s[k] == 2 || !(to_f32<T>(from[v]) > -INFINITY));
      const unsigned int found = __ballot_sync(0xffffffffu, is);
      const int at = have + __popc(found & ((1u << lane) - 1u));
      if (is && at < n_out) put(at, Candidate{score_bits(-INFINITY), make_key(0.f, ended ? p.pad_token : v), k});
      have += __popc(found);
    }
  }
  for (int at = have + lane; at < n_out; at += 32) put(at, Candidate{score_bits(-INFINITY), make_key(0.f, p.pad_token), 0});
}

// A slice of a row: `batch` pieces of 16 bytes per thread at a time, `batches` times.  The shortest that all go into one wave of blocks (kBePerSm per
// SM): a longer one takes longer, and one more wave too.  Measured, 80 rows of 50257 (fp32): 25 slices each 15.0 us, 7 slices 10.8.  The longest there is where none
// makes one wave.
struct Slicing {
  int batch, batches;
  int slices(const BeamProblem& p) const {
    const long long pieces = ((long long)p.vocab * (p.f32 ? 4 : 2) + 15) / 16, each = (long long)batch * batches * kBeThreads;
    return (int)((pieces + each - 1) / each);
  }
};
Slicing slicing(const BeamProblem& p, int sm_count) {
  for (const Slicing s : {Slicing{2, 1}, Slicing{4, 1}, Slicing{4, 2}, Slicing{4, 4}})
    if ((long long)p.batch * p.beams * s.slices(p) <= (long long)kBePerSm * sm_count) return s;
  return Slicing{4, 8};
}

template <typename T, bool kRagged> void (*pick(const Slicing& s))(BeamProblem, int, SliceStats*, u64*) {
  if (s.batch == 2) return beam_slice_kernel<T, 2, 1, kRagged>;
  switch (s.batches) {
    case 1: return beam_slice_kernel<T, 4, 1, kRagged>;
    case 2: return beam_slice_kernel<T, 4, 2, kRagged>;
    case 4: return beam_slice_kernel<T, 4, 4, kRagged>;
    default: return beam_slice_kernel<T, 4, 8, kRagged>;
  }
}

template <typename T>
cudaError_t launch_t(const BeamProblem& p, int sm_count, void* workspace, cudaStream_t st) {
  const Slicing s = slicing(p, sm_count);
  const int slices = s.slices(p);
  const long long blocks = (long long)p.batch * p.beams * slices;
  u64* const lists = (u64*)workspace;
  SliceStats* const stats = (SliceStats*)(lists + blocks * p.n_out);
  const bool ragged = rows_end_inside_a_piece((long long)p.batch * p.beams, p.stride, p.vocab, (int)sizeof(T));
  const cudaError_t e = launch_chained(ragged ? pick<T, true>(s) : pick<T, false>(s), dim3((unsigned int)blocks), kBeThreads, 0, st, p, slices, stats, lists);
  if (e != cudaSuccess) return e;
  return launch_chained(beam_join_kernel<T>, dim3((unsigned int)p.batch), kBeThreads, 0, st, p, slices, stats, lists);
}

}  // namespace

size_t beam_bytes(const BeamProblem& p, int sm_count) {
  return (size_t)p.batch * p.beams * slicing(p, sm_count).slices(p) * (p.n_out * sizeof(u64) + sizeof(SliceStats));
}

cudaError_t launch_beam_select(const BeamProblem& p, int sm_count, void* workspace, cudaStream_t st) {
  return p.f32 ? launch_t<float>(p, sm_count, workspace, st) : launch_t<__nv_bfloat16>(p, sm_count, workspace, st);
}

}  // namespace restkv
