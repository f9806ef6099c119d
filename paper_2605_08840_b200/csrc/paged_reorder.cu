// The cache of several hypotheses after a selection: tables in the order of the chosen parents, and the pages that have to be copied for it.
//
// Full pages are shared, so that a step moves what a hypothesis has of its last page at most, and only for those that do not go on in their
// parent's own: with c of B sequences childless, c last pages of a request.  A childless sequence's last page is nobody's any more, which
// makes it the place for a copy: no page is allocated, and none is both read and written.
//
// The tables: a thread per column takes it from all sequences of the request before it writes any (a table may be brought in order in
// place); who takes whose pages is found anew by every block, from `beams` parents in shared memory.  Bound by the table's bytes, and for
// one request by the launch.
// The pages: a block per copy, layer, K or V, and head, whose rows lie in one piece; blocks of sequences that copy nothing end at once.  40
// last pages of 8 layers, 46 MB read and as many written, take 17 us behind 4 for the tables, 5.4 TB/s; no unit is at its limit (issue slots 49%, L2 29%, DRAM
// 17%: copies of one page read it from L2 after the first, and what is written stays there), the blocks are short and begin with a load that the others wait
// for.  (A few larger blocks per page instead: the same there, 1 us more for one request.)
#include "paged.cuh"
#include "sm100_ptx.cuh"

namespace restkv {

namespace {

constexpr int kColumns = 128;       // of a block: a thread each
constexpr int kCopyThreads = 256;
constexpr int kMaxBeams = kBeamsMost;

// grid (column blocks, requests), dynamic shared memory: beams * kColumns entries
__global__ void __launch_bounds__(kColumns) paged_reorder_kernel(const PagedCache c, int beams, const int* __restrict__ parents, const int* table, int* table_out,
                                                                 int* __restrict__ copies, int* __restrict__ dropped) {
  extern __shared__ int column_s[];
  __shared__ int parent_s[kMaxBeams], donor_s[kMaxBeams];
  __shared__ unsigned int used_s[2], heir_s[2];          // bit per sequence: somebody goes on from it; it is the first to go on from its parent
  const int t = threadIdx.x, first = (int)blockIdx.y * beams;
  ptx::grid_dependency_wait();
  ptx::grid_dependency_launch();
  const int n = c.lengths[first];
  int parent = t;
  bool wrong = n < 0 || n > c.capacity();
  if (t < beams) {
    parent = parents[first + t];
    wrong |= (unsigned int)parent >= (unsigned int)beams || c.lengths[first + t] != n;
  }
  const bool bad = __syncthreads_or(wrong) != 0;
  if (bad) {                        // left as it is
    parent = t;
    if (t == 0 && blockIdx.x == 0) atomicOr(c.dev_status, kDevBadIndex);
  }
  if (t < beams) parent_s[t] = parent;
  __syncthreads();
  if (t < kMaxBeams) {
    bool used = false, heir = t < beams;
    for (int i = 0; i < beams; ++i) {
      const int p = parent_s[i];
      used |= p == t;
      heir &= i >= t || p != parent;
    }
    const unsigned int all_used = __ballot_sync(0xffffffffu, used), all_heirs = __ballot_sync(0xffffffffu, heir);
    if ((t & 31) == 0) { used_s[t >> 5] = all_used; heir_s[t >> 5] = all_heirs; }
  }
  __syncthreads();
  const unsigned long long used = used_s[0] | (unsigned long long)used_s[1] << 32, heirs = heir_s[0] | (unsigned long long)heir_s[1] << 32;
  if (t < beams) {
    int donor = parent;
    if (!(heirs >> t & 1)) {
      // the e-th sequence that does not take its parent's own takes those of the e-th that nobody goes on from: there are as many of both
      unsigned long long free = ~used;
      for (int left = t - __popcll(heirs & ((1ull << t) - 1)); left > 0; --left) free &= free - 1;
      donor = __ffsll((long long)free) - 1;
    }
    donor_s[t] = donor;
  }
  const int at = (int)blockIdx.x * kColumns + t, full = bad ? 0 : n / c.page_rows;
  const bool in = at < c.table_width;
  const long long base = (long long)first * c.table_width + at;
  for (int i = 0; i < beams; ++i)
    if (in) column_s[i * kColumns + t] = table[base + (long long)i * c.table_width];
  __syncthreads();
  if (blockIdx.x == 0 && t < beams) {
    const int rest = n - full * c.page_rows;
    const bool copy = !bad && donor_s[t] != parent && rest > 0;   // (rest > 0: the table has a column for them)
    int* const to = copies + 3ll * (first + t);
    to[2] = copy ? rest : 0;
    // the pages are another thread's column, and the table may be written below: looked up in the blocks that hold that column
    if (!copy) to[0] = to[1] = -1;
  }
  if (!in) return;
  if (at == full && !bad && n > full * c.page_rows) {
    for (int i = 0; i < beams; ++i)
      if (donor_s[i] != parent_s[i]) {
        const int src = column_s[parent_s[i] * kColumns + t], dst = column_s[donor_s[i] * kColumns + t];
        if ((unsigned int)src >= (unsigned int)c.n_pages || (unsigned int)dst >= (unsigned int)c.n_pages) atomicOr(c.dev_status, kDevBadIndex);
        copies[3ll * (first + i)] = src;
        copies[3ll * (first + i) + 1] = dst;
      }
  }
  for (int i = 0; i < beams; ++i) {
    const int from = at < full ? parent_s[i] : donor_s[i];
    if (from != i || table_out != table) table_out[base + (long long)i * c.table_width] = column_s[from * kColumns + t];
  }
  if (!dropped) return;
  for (int i = 0; i < beams; ++i) {
    const int page = column_s[i * kColumns + t];
    bool gone = at < full && !(used >> i & 1);
    for (int j = 0; gone && j < beams; ++j) gone = !(((used >> j & 1) || j < i) && column_s[j * kColumns + t] == page);
    dropped[base + (long long)i * c.table_width] = gone ? page : -1;
  }
}

// grid: copies x layers x 2 x heads, heads running fastest
__global__ void __launch_bounds__(kCopyThreads) paged_copy_kernel(const PagedCache c, const int* __restrict__ copies, int layers, long long layer_bytes, uint8_t* K_pages,
                                                                  uint8_t* V_pages) {
  unsigned int x = blockIdx.x;
  const int h = x % c.Hkv;
  x /= c.Hkv;
  const int side = x & 1;
  x >>= 1;
  const int layer = x % layers, i = x / layers;
  ptx::grid_dependency_wait();
  ptx::grid_dependency_launch();
  const int src = copies[3ll * i], dst = copies[3ll * i + 1], rows = copies[3ll * i + 2];
  if (src < 0 || src == dst || rows == 0) return;
  if (src >= c.n_pages || (unsigned int)dst >= (unsigned int)c.n_pages || rows < 0 || rows > c.page_rows) {
    if (threadIdx.x == 0) atomicOr(c.dev_status, kDevBadIndex);
    return;
  }
  uint8_t* const pool = (side ? V_pages : K_pages) + layer * layer_bytes;
  const long long page = (long long)c.Hkv * c.head_bytes, of_head = (long long)h * c.head_bytes;
  const uint4* __restrict__ from = reinterpret_cast<const uint4*>(pool + src * page + of_head);
  uint4* __restrict__ to = reinterpret_cast<uint4*>(pool + dst * page + of_head);
  const long long bytes = c.format == RESTKV_PAGES_INT4 ? (rows + kBlockRows - 1ll) / kBlockRows * c.block_bytes : (long long)rows * c.row_bytes;
  const long long all = bytes / 16;
  constexpr int kAhead = 4;
  for (long long k = threadIdx.x; k < all; k += kAhead * kCopyThreads) {
    uint4 v[kAhead];
#pragma unroll
    for (int y = 0; y < kAhead; ++y)
      if (k + y * kCopyThreads < all) v[y] = __ldcs(from + k + y * kCopyThreads);
#pragma unroll
    for (int y = 0; y < kAhead; ++y)
      if (k + y * kCopyThreads < all) to[k + y * kCopyThreads] = v[y];
  }
}

}  // namespace

cudaError_t launch_paged_reorder(const PagedCache& c, int beams, const int* parents, const int* table, int* table_out, int* copies, int* dropped, cudaStream_t st) {
  const dim3 grid((unsigned int)((c.table_width + kColumns - 1) / kColumns), (unsigned int)(c.batch / beams));
  return launch_chained(paged_reorder_kernel, grid, kColumns, (size_t)beams * kColumns * sizeof(int), st, c, beams, parents, table, table_out, copies, dropped);
}

cudaError_t launch_paged_copy(const PagedCache& c, const int* copies, int n_copies, int layers, long long layer_bytes, uint8_t* K_pages, uint8_t* V_pages, cudaStream_t st) {
  const long long blocks = (long long)n_copies * layers * 2 * c.Hkv;
  return launch_chained(paged_copy_kernel, dim3((unsigned int)blocks), kCopyThreads, 0, st, c, copies, layers, layer_bytes, K_pages, V_pages);
}

}  // namespace restkv
