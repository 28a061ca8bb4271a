// A server step's bookkeeping: pages of ended sequences onto the stack of free ones, pages, slots and positions for new tokens.
//
// One block sums the counts of all sequences up and writes what may be overwritten in place (lengths, the stack's size) when it
// has read it; with few rows it also moves the pages and writes the rows, with many a second launch does, whose blocks sum up
// again what the first has left (250000 rows of 1000 sequences: 28 us for release and plan where one block moves the pages). Bound:
// launches and chains of dependent reads (counts, sums, page numbers): 64 single tokens take 4.7 us, the release before them 3.7.
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
template <int WARPS>
__device__ __forceinline__ void block_scan(int64_t& a, int64_t& b, int64_t& all_a, int64_t& all_b) {
  __shared__ int64_t warp_a[32], warp_b[32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t a0 = a, b0 = b;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int64_t x = __shfl_up_sync(0xffffffffu, a, o), y = __shfl_up_sync(0xffffffffu, b, o);
    if (lane >= o) a += x, b += y;
  }
  if (lane == 31) warp_a[warp] = a, warp_b[warp] = b;
  __syncthreads();
  int64_t x = lane < WARPS ? warp_a[lane] : 0, y = lane < WARPS ? warp_b[lane] : 0;
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

// Lengths, rows and pages before each sequence, in shared memory.
struct Sums {
  int *len, *row, *page;
  int n_free, pages, rows;  // the stack's size, pages and rows in all
};
__device__ __forceinline__ int pages_of(const PlanParams& p, int n) { return n > 0 ? p.by_page.quot(n - 1) + 1 : 0; }  // (n <= 2^30)

// The pages that come: each warp of `warps` a run of them, a lane eight at a time (their numbers are on the way together).
__device__ __forceinline__ void take_pages(const PlanParams& p, const Sums& s, int warp, int warps) {
  const int n = s.pages, run = ((n + warps - 1) / warps + 31) / 32 * 32;
  const int64_t first = (int64_t)warp * run, end = min(first + run, (int64_t)n);
  int b = -1;
  for (int64_t i0 = first + (threadIdx.x & 31); i0 < end; i0 += 256) {
    const int32_t* from[8];
    int32_t* to[8];
    int id[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int64_t i64 = i0 + 32 * u;
      from[u] = nullptr;
      if (i64 >= end) continue;
      const int i = (int)i64;
      b = b < 0 ? owner(s.page, p.n_seqs, i) : walk(s.page, p.n_seqs, i, b);
      const int entry = pages_of(p, s.len[b]) + i - s.page[b], at = s.n_free - 1 - i;
      if (!in_bounds(entry, p.max_pages, p.status) || !in_bounds(at, p.free_capacity, p.status)) continue;
      int32_t* table = p.pages + (int64_t)b * p.max_pages + entry;
      from[u] = p.free_pages + at, to[u] = table;
      id[u] = *from[u];
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      if (from[u] == nullptr) continue;
      if (id[u] < 0 || id[u] >= p.n_pages) report(p.status, JAB_ERR_INVALID_ARG);
      *to[u] = id[u];
    }
  }
}

// The pages that go, in the same way, once all their numbers are known to be the cache's: else nothing is written and the answer is
// false. A warp's numbers stay in registers between the two where it has no more than 256 (8192 pages in all). Called by the whole block.
__device__ __forceinline__ bool give_pages(const PlanParams& p, const Sums& s, int warp, int warps) {
  const int n = s.pages, run = ((n + warps - 1) / warps + 31) / 32 * 32, same = p.shared / p.page;
  const int64_t first = (int64_t)warp * run, end = min(first + run, (int64_t)n), begin = first + (threadIdx.x & 31);
  int b = -1, id[8];
  auto fetch = [&](int64_t i0) {
    bool fine = true;
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int64_t i64 = i0 + 32 * u;
      id[u] = 0;
      if (i64 >= end) continue;
      const int i = (int)i64;
      b = b < 0 ? owner(s.page, p.n_seqs, i) : walk(s.page, p.n_seqs, i, b);
      const int entry = same + i - s.page[b];
      if (in_bounds(entry, p.max_pages, p.status)) id[u] = p.pages[(int64_t)b * p.max_pages + entry];
    }
#pragma unroll
    for (int u = 0; u < 8; ++u) fine = fine && id[u] >= 0 && id[u] < p.n_pages;
    return fine;
  };
  bool fine = true;
  for (int64_t i0 = begin; i0 < end; i0 += 256) fine = fetch(i0) && fine;
  if (!__syncthreads_and(fine)) return false;
  b = -1;
  for (int64_t i0 = begin; i0 < end; i0 += 256) {
    if (run > 256) fetch(i0);
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int64_t i = i0 + 32 * u;
      if (i < end && in_bounds(s.n_free + i, p.free_capacity, p.status)) p.free_pages[s.n_free + i] = id[u];
    }
  }
  return true;
}

// Slots and positions of all rows, padding behind the last: as above, four rows of a lane at a time.
__device__ __forceinline__ void write_rows(const PlanParams& p, const Sums& s, int warp, int warps) {
  const int n = (int)p.n_tokens, run = ((n + warps - 1) / warps + 31) / 32 * 32;
  const int64_t first = (int64_t)warp * run, end = min(first + run, (int64_t)n);
  int b = -1;
  for (int64_t i0 = first + (threadIdx.x & 31); i0 < end; i0 += 128) {
    int pos[4], id[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int64_t i = i0 + 32 * u;
      pos[u] = 0, id[u] = -1;
      if (i >= end || i >= s.rows) continue;
      b = b < 0 ? owner(s.row, p.n_seqs, (int)i) : walk(s.row, p.n_seqs, (int)i, b);
      pos[u] = s.len[b] + (int)i - s.row[b];
      // a page of this call comes from the stack: its entry may not be written yet
      const int entry = p.by_page.quot(pos[u]), mine = pages_of(p, s.len[b]);
      id[u] = entry < mine ? p.pages[(int64_t)b * p.max_pages + entry] : p.free_pages[s.n_free - 1 - s.page[b] - (entry - mine)];
      if (id[u] < 0 || id[u] >= p.n_pages) report(p.status, JAB_ERR_INVALID_ARG), id[u] = -1;
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int64_t i = i0 + 32 * u;
      if (i >= end || !in_bounds(i, p.n_tokens, p.status)) continue;
      p.positions[i] = pos[u];
      p.slots[i] = id[u] < 0 ? -1 : (int64_t)id[u] * p.page + pos[u] - p.by_page.quot(pos[u]) * p.page;
    }
  }
}

// RELEASE: counts says which sequences have ended. Else counts of new tokens.
template <bool RELEASE>
__global__ void __launch_bounds__(kThreads, 1) kv_plan_kernel(const __grid_constant__ PlanParams p) {
  extern __shared__ int smem[];
  int *len_s = smem, *row_s = len_s + p.n_seqs, *page_s = row_s + p.n_seqs;  // [n_seqs] each
  __shared__ int bad_s;
  if (threadIdx.x == 0) bad_s = 0;
  stream_order();
  __syncthreads();
  const int tid = threadIdx.x;
  const int each = (p.n_seqs + kThreads - 1) / kThreads, b0 = min(tid * each, p.n_seqs), b1 = min(b0 + each, p.n_seqs);
  const int64_t room = (int64_t)p.max_pages * p.page;
  const int n_free = *p.n_free;
  const int same = RELEASE ? p.shared / p.page : 0;
  auto pages_for = [&](int len, int count) {  // that come or go
    return RELEASE ? (count != 0 ? max(pages_of(p, len) - same, 0) : 0) : pages_of(p, len + count) - pages_of(p, len);
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
  block_scan<kWarps>(rows, pages, all_rows, all_pages);
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
  Sums sums{len_s, row_s, page_s, n_free, bad ? 0 : (int)all_pages, bad ? 0 : (int)all_rows};
  if (RELEASE && !bad) bad = !give_pages(p, sums, tid >> 5, kWarps);
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
  if (RELEASE || p.n_tokens > kRowsInOne) return;
  take_pages(p, sums, tid >> 5, kWarps);
  write_rows(p, sums, tid >> 5, kWarps);
}

// Pages and rows behind a first launch that did the rest (a call that it refused has no rows).
__global__ void __launch_bounds__(kRowThreads) kv_rows_kernel(const __grid_constant__ PlanParams p) {
  extern __shared__ int smem[];
  int *len_s = smem, *row_s = len_s + p.n_seqs, *page_s = row_s + p.n_seqs;
  stream_order();
  const int tid = threadIdx.x, each = (p.n_seqs + kRowThreads - 1) / kRowThreads, b0 = min(tid * each, p.n_seqs), b1 = min(b0 + each, p.n_seqs);
  int64_t none = 0, pages = 0, all_none, all_pages;
  auto pages_for = [&](int b, int& len) {
    const int count = p.q_start[b + 1] - p.q_start[b], now = p.new_lens[b];
    len = now - count;
    return count > 0 ? pages_of(p, now) - pages_of(p, len) : 0;
  };
  for (int b = b0; b < b1; ++b) {
    int len;
    pages += pages_for(b, len);
    len_s[b] = len, row_s[b] = p.q_start[b];
  }
  block_scan<kRowThreads / 32>(none, pages, all_none, all_pages);
  for (int b = b0; b < b1; ++b) {
    int len;
    page_s[b] = (int)pages;
    pages += pages_for(b, len);
  }
  __syncthreads();
  const Sums sums{len_s, row_s, page_s, *p.new_free + (int)all_pages, (int)all_pages, p.q_start[p.n_seqs]};
  const int warp = blockIdx.x * (kRowThreads / 32) + (tid >> 5), warps = gridDim.x * (kRowThreads / 32);
  take_pages(p, sums, warp, warps);
  write_rows(p, sums, warp, warps);
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
  e = ready.once(dev, [&] {
    const cudaError_t f = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, 3 * kMostSeqs * 4);
    return f != cudaSuccess ? f : cudaFuncSetAttribute(kv_rows_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 3 * kMostSeqs * 4);
  });
  if (e != cudaSuccess) return e;
  e = launch_after(kern, 1u, kThreads, (size_t)3 * a.n_seqs * 4, st, p);
  if (e != cudaSuccess || RELEASE || a.n_tokens <= kRowsInOne) return e;
  return launch_after(kv_rows_kernel, (unsigned)((a.n_tokens + kRowsPerBlock - 1) / kRowsPerBlock), kRowThreads, (size_t)3 * a.n_seqs * 4, st, p);
}

}  // namespace

int kv_plan_kernels(const KvPlanArgs& a) { return a.n_tokens > kRowsInOne ? 2 : 1; }
cudaError_t launch_kv_plan(const KvPlanArgs& a, cudaStream_t st) { return launch<false>(a, st); }
cudaError_t launch_kv_release(const KvPlanArgs& a, cudaStream_t st) { return launch<true>(a, st); }

}  // namespace jab
