// A server step's bookkeeping: pages of ended sequences onto the stack of free ones, pages, slots and positions for new tokens.
//
// One block sums the counts of all sequences up, moves the pages and writes what may be overwritten in place (lengths, the
// stack's size) when it has read it; with few rows it writes those too, with many a second launch does, from the starts,
// lengths and page tables that the first has left. Bound: launches and chains of dependent reads (counts, sums, page numbers):
// 64 single tokens take 3.9 us.
#include <algorithm>

#include "common.cuh"
#include "per_device.h"
#include "serve.h"
#include "tc.cuh"

namespace jab {
namespace {

constexpr int kThreads = 1024, kWarps = kThreads / 32;
constexpr int kMostSeqs = 8192;
constexpr int kRowsInOne = 4096;   // rows that the first launch writes itself
constexpr int kRowThreads = 256, kRowsPerBlock = 2048;

struct PlanParams {
  int n_seqs, page, max_pages, free_capacity, shared;
  FastDiv by_page;
  int64_t n_pages, n_tokens;
  const int32_t *lens, *counts, *n_free;
  int32_t *pages, *free_pages, *new_lens, *new_free, *q_start, *positions;
  int64_t* slots;
  int* status;
};

// Sums over the block's threads before this one (a, b) and over all of them (all_a, all_b).
__device__ __forceinline__ void block_scan(int64_t& a, int64_t& b, int64_t& all_a, int64_t& all_b) {
  __shared__ int64_t warp_a[kWarps], warp_b[kWarps];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t a0 = a, b0 = b;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t x = __shfl_up_sync(0xffffffffu, a, o), y = __shfl_up_sync(0xffffffffu, b, o);
    if (lane >= o) a += x, b += y;
  }
  if (lane == 31) warp_a[warp] = a, warp_b[warp] = b;
  __syncthreads();
  int64_t x = warp_a[lane], y = warp_b[lane];
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t u = __shfl_up_sync(0xffffffffu, x, o), v = __shfl_up_sync(0xffffffffu, y, o);
    if (lane >= o) x += u, y += v;
  }
  all_a = __shfl_sync(0xffffffffu, x, 31), all_b = __shfl_sync(0xffffffffu, y, 31);
  const int64_t pa = __shfl_sync(0xffffffffu, x, max(warp - 1, 0)), pb = __shfl_sync(0xffffffffu, y, max(warp - 1, 0));
  a += (warp > 0 ? pa : 0) - a0, b += (warp > 0 ? pb : 0) - b0;
}

// The last b with start[b] <= i (start[0] = 0 <= i), from `b` on.
__device__ __forceinline__ int owner(const int* start, int n, int i) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (start[mid] <= i) lo = mid;
    else hi = mid;
  }
  return lo;
}
// The same for a larger i than the one that gave b: a few steps on, or a search of the rest (many sequences of a token each).
__device__ __forceinline__ int walk(const int* start, int n, int i, int b) {
#pragma unroll 1
  for (int k = 0; k < 4; ++k) {
    if (b + 1 >= n || start[b + 1] > i) return b;
    ++b;
  }
  return b + owner(start + b, n - b, i);
}

// Slots and positions of the rows [first, end), those from `real` on padding: a warp takes a run of them, a lane four at a time (their
// page numbers are on the way together). page(b, row, position&) is the page number of sequence b's row.
template <class Page>
__device__ __forceinline__ void rows_of(const PlanParams& p, int tid, int threads, int first, int end, int real, const int* start, Page page) {
  const int warps = threads / 32, run = ((end - first + warps - 1) / warps + 31) / 32 * 32;
  const int64_t from = first + (int64_t)(tid >> 5) * run, to = min(from + run, (int64_t)end);
  int b = -1;
  for (int64_t i0 = from + (tid & 31); i0 < to; i0 += 128) {
    int pos[4], id[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int64_t i = i0 + 32 * u;
      pos[u] = 0, id[u] = -1;
      if (i >= to || i >= real) continue;
      b = b < 0 ? owner(start, p.n_seqs, (int)i) : walk(start, p.n_seqs, (int)i, b);
      id[u] = page(b, (int)i, pos[u]);
      if (id[u] < 0 || id[u] >= p.n_pages) report(p.status, JAB_ERR_INVALID_ARG), id[u] = -1;
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int64_t i = i0 + 32 * u;
      if (i >= to || !in_bounds(i, p.n_tokens, p.status)) continue;
      p.positions[i] = pos[u];
      p.slots[i] = id[u] < 0 ? -1 : (int64_t)id[u] * p.page + pos[u] - p.by_page.quot(pos[u]) * p.page;
    }
  }
}

// RELEASE: counts says which sequences have ended. Else counts of new tokens.
template <bool RELEASE>
__global__ void __launch_bounds__(kThreads, 1) kv_plan_kernel(const __grid_constant__ PlanParams p) {
  extern __shared__ int smem[];
  int* len_s = smem;                    // [n_seqs]
  int* row_s = len_s + p.n_seqs;        // rows before a sequence [n_seqs]
  int* page_s = row_s + p.n_seqs;       // pages given or taken before a sequence [n_seqs]
  __shared__ int bad_s;
  if (threadIdx.x == 0) bad_s = 0;
  stream_order();
  __syncthreads();
  const int tid = threadIdx.x;
  const int each = (p.n_seqs + kThreads - 1) / kThreads, b0 = min(tid * each, p.n_seqs), b1 = min(b0 + each, p.n_seqs);
  const int64_t room = (int64_t)p.max_pages * p.page;
  const int n_free = *p.n_free;
  const int same = RELEASE ? p.shared / p.page : 0;
  auto pages_of = [&](int n) { return n > 0 ? p.by_page.quot(n - 1) + 1 : 0; };  // (n <= 2^30)
  auto pages_for = [&](int len, int count) {  // that come or go
    return RELEASE ? (count != 0 ? max(pages_of(len) - same, 0) : 0) : pages_of(len + count) - pages_of(len);
  };
  int64_t rows = 0, pages = 0;
  bool bad = n_free < 0 || n_free > p.free_capacity;
  for (int b = b0; b < b1; ++b) {
    const int len = p.lens[b], count = p.counts[b];
    if (len < 0 || len > room || (!RELEASE && (count < 0 || (int64_t)len + count > room))) {
      bad = true;
      continue;
    }
    len_s[b] = len;
    rows += RELEASE ? 0 : count;
    pages += pages_for(len, count);
  }
  int64_t all_rows, all_pages;
  if (bad) bad_s = 1;  // (any thread's word)
  block_scan(rows, pages, all_rows, all_pages);
  bad = bad_s != 0 || all_rows > p.n_tokens || (RELEASE ? n_free + all_pages > p.free_capacity : all_pages > n_free);
  int64_t r = rows, g = pages;
  if (!bad)
    for (int b = b0; b < b1; ++b) {
      const int count = p.counts[b];
      row_s[b] = (int)r, page_s[b] = (int)g;
      r += RELEASE ? 0 : count;
      g += pages_for(len_s[b], count);
    }
  __syncthreads();
  // (in place: every thread has read the stack's size, and a sequence's length and count are read by one thread alone)
  for (int b = b0; b < b1; ++b) {
    int to;
    if (RELEASE) {
      const int len = p.lens[b];
      to = !bad && p.counts[b] != 0 ? min(len, p.shared) : len;
    } else {
      to = bad ? p.lens[b] : len_s[b] + p.counts[b];
      p.q_start[b] = bad ? 0 : row_s[b];
    }
    p.new_lens[b] = to;
  }
  if (tid == 0) {
    *p.new_free = bad ? n_free : RELEASE ? n_free + (int)all_pages : n_free - (int)all_pages;
    if (!RELEASE) p.q_start[p.n_seqs] = bad ? 0 : (int)all_rows;
    if (bad) report(p.status, JAB_ERR_INVALID_ARG);
  }
  const int lane = tid & 31, warp = tid >> 5;
  // pages that come or go: a warp takes a run of them
  if (!bad && all_pages > 0) {
    const int n = (int)all_pages, run = ((n + kWarps - 1) / kWarps + 31) / 32 * 32;
    const int64_t first = (int64_t)warp * run;
    int b = -1;
    for (int64_t i64 = first + lane; i64 < min(first + run, (int64_t)n); i64 += 32) {
      const int i = (int)i64;
      b = b < 0 ? owner(page_s, p.n_seqs, i) : walk(page_s, p.n_seqs, i, b);
      const int entry = (RELEASE ? same : pages_of(len_s[b])) + i - page_s[b];
      int32_t* at = p.pages + (int64_t)b * p.max_pages + entry;
      int32_t* stack = p.free_pages + (RELEASE ? n_free + i : n_free - 1 - i);
      const int id = RELEASE ? *at : *stack;
      if (id < 0 || id >= p.n_pages) report(p.status, JAB_ERR_INVALID_ARG);
      if (RELEASE)
        *stack = id;
      else
        *at = id;
    }
  }
  if (RELEASE || p.n_tokens > kRowsInOne) return;
  // a page of this call comes from the stack: its entry may not be written yet
  const int real = bad ? 0 : (int)all_rows;
  rows_of(p, tid, kThreads, 0, (int)p.n_tokens, real, row_s, [&](int b, int i, int& pos) {
    pos = len_s[b] + i - row_s[b];
    const int entry = p.by_page.quot(pos), mine = pages_of(len_s[b]);
    return entry < mine ? p.pages[(int64_t)b * p.max_pages + entry] : p.free_pages[n_free - 1 - page_s[b] - (entry - mine)];
  });
}

__global__ void __launch_bounds__(kRowThreads) kv_rows_kernel(const __grid_constant__ PlanParams p) {
  extern __shared__ int start[];  // [n_seqs + 1]
  stream_order();
  for (int b = threadIdx.x; b <= p.n_seqs; b += kRowThreads) start[b] = p.q_start[b];
  __syncthreads();
  const int first = blockIdx.x * kRowsPerBlock, end = min(first + kRowsPerBlock, (int)p.n_tokens);
  rows_of(p, threadIdx.x, kRowThreads, first, end, min(start[p.n_seqs], end), start, [&](int b, int i, int& pos) {
    pos = p.new_lens[b] - (start[b + 1] - i);
    return p.pages[(int64_t)b * p.max_pages + p.by_page.quot(pos)];
  });
}

template <bool RELEASE>
cudaError_t launch(const KvPlanArgs& a, cudaStream_t st) {
  PlanParams p{};
  p.n_seqs = a.n_seqs, p.page = a.page, p.max_pages = a.max_pages, p.free_capacity = a.free_capacity, p.shared = a.shared;
  p.n_pages = a.n_pages, p.n_tokens = a.n_tokens;
  p.lens = a.lens, p.counts = a.counts, p.n_free = a.n_free;
  p.pages = a.pages, p.free_pages = a.free_pages, p.new_lens = a.new_lens, p.new_free = a.new_free;
  p.q_start = a.q_start, p.positions = a.positions, p.slots = a.slots;
  p.by_page = FastDiv(a.page);
  p.status = a.status;
  auto kern = kv_plan_kernel<RELEASE>;
  static SetUp ready;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  e = ready.once(dev, [&] { return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, 3 * kMostSeqs * 4); });
  if (e != cudaSuccess) return e;
  e = launch_after(kern, 1u, kThreads, (size_t)3 * a.n_seqs * 4, st, p);
  if (e != cudaSuccess || RELEASE || a.n_tokens <= kRowsInOne) return e;
  return launch_after(kv_rows_kernel, (unsigned)((a.n_tokens + kRowsPerBlock - 1) / kRowsPerBlock), kRowThreads, (size_t)(a.n_seqs + 1) * 4, st, p);
}

}  // namespace

int kv_plan_kernels(const KvPlanArgs& a) { return a.n_tokens > kRowsInOne ? 2 : 1; }
cudaError_t launch_kv_plan(const KvPlanArgs& a, cudaStream_t st) { return launch<false>(a, st); }
cudaError_t launch_kv_release(const KvPlanArgs& a, cudaStream_t st) { return launch<true>(a, st); }

}  // namespace jab
