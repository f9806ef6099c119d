// The best continuations of a request's hypotheses: scores[k] + logits[k,v] - log sum exp(logits[k,:]), over hypotheses and tokens.
//
// One pass over the logits.  A block has a slice of a row in registers: its maximum and sum of exponentials, and its n_out largest logits.  A
// second kernel joins a request's slices: normalisers, scores in 64 bits, the n_out best.
// Largest of a block: groups of four threads name their largest logit; the n_out-th of those bounds the n_out-th of the slice from below, and
// what reaches it, a few more than n_out as a rule, goes to shared memory and is ranked by counting.  Where it is more than the list holds
// (a slice of equal logits, say) the largest are taken one by one instead.  The second kernel does the same with scores.
// Logits of -inf are no candidates in either; requests that run out of others look for them in the rows at the end.
// What bounds it: HBM for large calls, beside it the special-function unit (an exponential per logit: 16 per clock and SM, 14 us for the
// 67 million logits of 512 rows of 131072 whose bytes take 21); for small ones two launches, each a chain of loads and a few barriers.
#include <math.h>

#include "beam.cuh"
#include "sm100_ptx.cuh"

namespace restkv {

namespace {

using namespace ptx;

constexpr int kBeThreads = 256, kBeWarps = kBeThreads / 32;
constexpr int kGroups = kBeThreads / 4;         // at least kBeamOut
constexpr int kList = 1024;
constexpr float kLog2e = 1.4426950408889634f;
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

// The n-th largest of the groups' values, of kGroups by their first threads; ends with a barrier.
__device__ __forceinline__ float nth_of_groups(float mine, int n, float (&group_s)[kGroups], float& limit_s) {
  const int t = threadIdx.x;
  mine = fmaxf(mine, __shfl_xor_sync(0xffffffffu, mine, 1));
  mine = fmaxf(mine, __shfl_xor_sync(0xffffffffu, mine, 2));
  if ((t & 3) == 0) group_s[t >> 2] = mine;
  __syncthreads();
  if (t < kGroups) {
    const float x = group_s[t];
    int before = 0;
#pragma unroll
    for (int i = 0; i < kGroups; i += 4) {
      const float4 y = *reinterpret_cast<const float4*>(&group_s[i]);
      before += (y.x > x || (y.x == x && i < t)) + (y.y > x || (y.y == x && i + 1 < t)) + (y.z > x || (y.z == x && i + 2 < t)) + (y.w > x || (y.w == x && i + 3 < t));
    }
    if (before == n - 1) limit_s = x;
  }
  __syncthreads();
  return limit_s;
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

struct SliceStats { float top, sum; };   // of a slice: its maximum and the sum of exp(x - top); no finite logit: -inf, 0

// grid: rows x slices, slices running fastest.  A slice is kVec * kBeThreads pieces of 16 bytes of a row.
template <typename T, int kVec>
__global__ void __launch_bounds__(kBeThreads) beam_slice_kernel(const BeamProblem p, int slices, SliceStats* __restrict__ stats, u64* __restrict__ lists) {
  using V = Vec<T>;
  constexpr int kPer = V::kPer;
  __shared__ __align__(16) float group_s[kGroups];
  __shared__ float limit_s, top_s[kBeWarps], sum_s[kBeWarps];
  __shared__ int count_s;
  __shared__ u64 list_s[kList], best_s[kBeWarps];
  const int row = blockIdx.x / slices, slice = blockIdx.x - row * slices, t = threadIdx.x, lane = t & 31, warp = t >> 5;
  grid_dependency_wait();
  grid_dependency_launch();
  if (row_kind(p, row) != 0) return;
  const T* const from = reinterpret_cast<const T*>(p.logits) + row * p.stride;
  // A thread's tokens do not depend on where in its 16-byte pieces the row begins: equal rows have equal sums, bit for bit.
  const unsigned int off = (unsigned int)(reinterpret_cast<uintptr_t>(from) & 15u);   // bytes of the row before in the row's first piece
  const uint4* const pieces = reinterpret_cast<const uint4*>(reinterpret_cast<uintptr_t>(from) & ~(uintptr_t)15);
  const int piece0 = slice * (kVec * kBeThreads) + t, in_row = (int)(((long long)p.vocab * (int)sizeof(T) + off + 15) / 16);
  auto token_of = [&](int y, int i) { return (piece0 + y * kBeThreads) * kPer + i; };
  V v[kVec];
#pragma unroll
  for (int y = 0; y < kVec; ++y) v[y].u = piece0 + y * kBeThreads < in_row ? __ldcs(pieces + piece0 + y * kBeThreads) : make_uint4(0u, 0u, 0u, 0u);
  if (off) {
#pragma unroll
    for (int y = 0; y < kVec; ++y) {
      uint4 next = make_uint4(__shfl_down_sync(0xffffffffu, v[y].u.x, 1), __shfl_down_sync(0xffffffffu, v[y].u.y, 1), __shfl_down_sync(0xffffffffu, v[y].u.z, 1),
                              __shfl_down_sync(0xffffffffu, v[y].u.w, 1));
      if (lane == 31) next = piece0 + y * kBeThreads + 1 < in_row ? __ldcs(pieces + piece0 + y * kBeThreads + 1) : make_uint4(0u, 0u, 0u, 0u);
      v[y].u = shifted(v[y].u, next, off);
    }
  }
#pragma unroll
  for (int y = 0; y < kVec; ++y) {
    if (token_of(y, kPer) <= p.vocab) continue;
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (token_of(y, i) >= p.vocab) v[y].set(i, -INFINITY);
  }
  if (t == 0) count_s = 0;
  float top = -INFINITY;                                                // (a NaN is passed over)
#pragma unroll
  for (int y = 0; y < kVec; ++y)
#pragma unroll
    for (int i = 0; i < kPer; i += 2) top = fmax3(top, v[y].at(i), v[y].at(i + 1));
  auto sum_by = [&](float of, auto&& value) {
    f32x2 s0 = f2_make(0.f, 0.f), s1 = s0;
    const f32x2 minus = f2_make(-of, -of), scale = f2_make(kLog2e, kLog2e);
#pragma unroll
    for (int y = 0; y < kVec; ++y)
#pragma unroll
      for (int i = 0; i < kPer; i += 4) {
        // the difference first: large terms have small ones, whose rounding is small
        const f32x2 a = f2_mul(f2_add(f2_make(value(v[y].at(i)), value(v[y].at(i + 1))), minus), scale);
        const f32x2 b = f2_mul(f2_add(f2_make(value(v[y].at(i + 2)), value(v[y].at(i + 3))), minus), scale);
        s0 = f2_add(s0, f2_make(ex2_approx(f2_lo(a)), ex2_approx(f2_hi(a))));
        s1 = f2_add(s1, f2_make(ex2_approx(f2_lo(b)), ex2_approx(f2_hi(b))));
      }
    s0 = f2_add(s0, s1);
    return f2_lo(s0) + f2_hi(s0);
  };
  float sum = sum_by(top == -INFINITY ? 0.f : top, [](float x) { return x; });
  // A NaN or +inf among the logits shows in the sum, and all is made again of what counts in their place.
  const bool odd = !(sum < INFINITY);
  if (odd) {
    top = usable(top);
    sum = sum_by(top == -INFINITY ? 0.f : top, [](float x) { return usable(x); });
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
  // ---- what reaches the limit ----
  if (top >= limit && top > -INFINITY) {
#pragma unroll
    for (int y = 0; y < kVec; ++y)
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const float x = v[y].at(i);
        // (a NaN compares false; +inf is above every limit)
        if (x >= limit && x > -INFINITY) {
          const int at = atomicAdd(&count_s, 1);
          if (at < kList) list_s[at] = make_key(usable(x), token_of(y, i));
        }
      }
  }
  __syncthreads();
  const int count = count_s;
  u64* const list = lists + (long long)blockIdx.x * p.n_out;
  if (count <= kList) {
    for (int x = t; x < count; x += kBeThreads) {
      const u64 mine = list_s[x];
      int before = 0;
      for (int y = 0; y < count; ++y) before += list_s[y] > mine;
      if (before < p.n_out) list[before] = mine;
    }
    for (int x = count + t; x < p.n_out; x += kBeThreads) list[x] = 0;
  } else {
    u64 last = ~0ull;
    for (int k = 0; k < p.n_out; ++k) {
      u64 best = 0;
#pragma unroll
      for (int y = 0; y < kVec; ++y)
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
          const float x = v[y].at(i);
          if (!(x > -INFINITY)) continue;
          const u64 key = make_key(usable(x), token_of(y, i));
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
      if (t == 0) list[k] = last;             // (more than kList candidates: never 0)
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

// A continuation by its score, hypothesis and key.
struct Candidate {
  double score;
  u64 key;
  int beam;
  __device__ bool before(const Candidate& o) const { return score > o.score || (score == o.score && (beam < o.beam || (beam == o.beam && key > o.key))); }
};

// grid: requests
template <typename T>
__global__ void __launch_bounds__(kBeThreads) beam_join_kernel(const BeamProblem p, int slices, const SliceStats* __restrict__ stats, const u64* __restrict__ lists) {
  __shared__ __align__(16) float group_s[kGroups];
  __shared__ float limit_s;
  __shared__ int count_s, kind_s[kBeamsPerRequest];
  __shared__ double score_s[kBeamsPerRequest], total_s[kBeamsPerRequest];   // hypotheses' scores and normalisers
  __shared__ Candidate list_s[kList / 2], best_s[kBeWarps];
  const int t = threadIdx.x, lane = t & 31, warp = t >> 5, row0 = (int)blockIdx.x * p.beams, n_out = p.n_out;
  grid_dependency_wait();
  grid_dependency_launch();
  if (t == 0) count_s = 0;
  for (int k = warp; k < p.beams; k += kBeWarps) {
    const int row = row0 + k, kind = row_kind(p, row);
    double total = 0.0;
    if (kind == 0) {
      float m = -INFINITY;
      for (int x = lane; x < slices; x += 32) m = fmaxf(m, __ldcg(&stats[(long long)row * slices + x].top));
#pragma unroll
      for (int x = 16; x > 0; x >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, x));
      double s = 0.0;
      for (int x = lane; x < slices; x += 32) {
        const float top = __ldcg(&stats[(long long)row * slices + x].top), sum = __ldcg(&stats[(long long)row * slices + x].sum);
        if (top > -INFINITY) s += (double)sum * (double)ex2_approx((top - m) * kLog2e);
      }
#pragma unroll
      for (int x = 16; x > 0; x >>= 1) s += __shfl_xor_sync(0xffffffffu, s, x);
      total = (double)m + log(s);                 // (a row without candidates has none that would use it)
    }
    if (lane == 0) { kind_s[k] = kind; score_s[k] = (double)p.scores[row]; total_s[k] = total; }
  }
  __syncthreads();
  // candidate x of the request: hypotheses one after the other, each with the lists of its slices
  const int per_row = slices * n_out, all = p.beams * per_row;
  auto candidate = [&](int x) {
    const int k = x / per_row, y = x - k * per_row, kind = kind_s[k];
    Candidate c{0.0, 0, k};
    if (kind == 0) {
      c.key = __ldcg(lists + (long long)(row0 + k) * per_row + y);
      c.score = score_s[k] + ((double)key_logit(c.key) - total_s[k]);
    } else if (kind == 1 && y == 0) {
      c.key = make_key(0.f, p.pad_token);
      c.score = score_s[k];
    }
    return c;
  };
  float top = -INFINITY;
  for (int x = t; x < all; x += kBeThreads) {
    const Candidate c = candidate(x);
    if (c.key) top = fmaxf(top, (float)c.score);
  }
  const float limit = nth_of_groups(top, n_out, group_s, limit_s);
  for (int x = t; x < all; x += kBeThreads) {
    const Candidate c = candidate(x);
    if (!c.key || !((float)c.score >= limit)) continue;
    const int at = atomicAdd(&count_s, 1);
    if (at < kList / 2) list_s[at] = c;
  }
  __syncthreads();
  const int count = count_s;
  auto put = [&](int at, const Candidate& c) {
    const long long to = (long long)blockIdx.x * n_out + at;
    p.parents[to] = c.beam;
    p.tokens[to] = key_token(c.key);
    p.scores_out[to] = (float)c.score;
  };
  if (count <= kList / 2) {
    for (int x = t; x < count; x += kBeThreads) {
      const Candidate mine = list_s[x];
      int before = 0;
      for (int y = 0; y < count; ++y) before += list_s[y].before(mine);
      if (before < n_out) put(before, mine);
    }
  } else {
    Candidate last{INFINITY, ~0ull, -1};
    for (int k = 0; k < n_out; ++k) {
      Candidate best{0.0, 0, 0};                  // key 0: none
      for (int x = t; x < all; x += kBeThreads) {
        const Candidate c = candidate(x);
        if (c.key && last.before(c) && (!best.key || c.before(best))) best = c;
      }
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
      if (is && at < n_out) put(at, Candidate{-INFINITY, make_key(0.f, ended ? p.pad_token : v), k});
      have += __popc(found);
    }
  }
  for (int at = have + lane; at < n_out; at += 32) put(at, Candidate{-INFINITY, make_key(0.f, p.pad_token), 0});
}

// 16-byte pieces of a row for a thread: many where there are blocks enough, else few, for more blocks.
int vectors(const BeamProblem& p, int sm_count) {
  const long long rows = (long long)p.batch * p.beams, pieces = ((long long)p.vocab * (p.f32 ? 4 : 2) + 15) / 16;
  return rows * ((pieces + 8 * kBeThreads - 1) / (8 * kBeThreads)) < 2 * sm_count ? 2 : 8;
}
int slices_of(const BeamProblem& p, int vec) {
  const long long pieces = ((long long)p.vocab * (p.f32 ? 4 : 2) + 15) / 16;
  return (int)((pieces + (long long)vec * kBeThreads - 1) / ((long long)vec * kBeThreads));
}

template <typename T>
cudaError_t launch_t(const BeamProblem& p, int sm_count, void* workspace, cudaStream_t st) {
  const int vec = vectors(p, sm_count), slices = slices_of(p, vec);
  const long long blocks = (long long)p.batch * p.beams * slices;
  u64* const lists = (u64*)workspace;
  SliceStats* const stats = (SliceStats*)(lists + blocks * p.n_out);
  const auto kernel = vec == 2 ? beam_slice_kernel<T, 2> : beam_slice_kernel<T, 8>;
  const cudaError_t e = launch_chained(kernel, dim3((unsigned int)blocks), kBeThreads, 0, st, p, slices, stats, lists);
  if (e != cudaSuccess) return e;
  return launch_chained(beam_join_kernel<T>, dim3((unsigned int)p.batch), kBeThreads, 0, st, p, slices, stats, lists);
}

}  // namespace

size_t beam_bytes(const BeamProblem& p, int sm_count) {
  return (size_t)p.batch * p.beams * slices_of(p, vectors(p, sm_count)) * (p.n_out * sizeof(u64) + sizeof(SliceStats));
}

cudaError_t launch_beam_select(const BeamProblem& p, int sm_count, void* workspace, cudaStream_t st) {
  return p.f32 ? launch_t<float>(p, sm_count, workspace, st) : launch_t<__nv_bfloat16>(p, sm_count, workspace, st);
}

}  // namespace restkv
