// A server step's bookkeeping: pages of ended sequences onto the stack of free ones, pages, slots and positions for new tokens.
//
// One cluster does a call: every block sums the counts of all sequences up for itself (8 bytes a sequence, from L2), then takes
// its share of the rows and pages; what may be overwritten in place (lengths, the stack's size) is written behind the
// cluster's barrier, when all blocks have read it. Bound: the launch and a chain of three dependent reads (counts, sums,
// page numbers) for a decoding step; stores of 12 bytes a row for long prompts.
#include <algorithm>

#include "common.cuh"
#include "per_device.h"
#include "serve.h"
#include "tc.cuh"

namespace jab {
namespace {

constexpr int kThreads = 1024, kWarps = kThreads / 32;
constexpr int kMostSeqs = 8192;
constexpr int kMostBlocks = 8;      // of the cluster
constexpr int kRowsPerBlock = 8192;  // from where one more block pays

struct PlanParams {
  int n_seqs, page, max_pages, free_capacity, shared;
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
  const int blocks = gridDim.x, rank = blockIdx.x, tid = threadIdx.x;
  const int each = (p.n_seqs + kThreads - 1) / kThreads, b0 = min(tid * each, p.n_seqs), b1 = min(b0 + each, p.n_seqs);
  const int64_t room = (int64_t)p.max_pages * p.page;
  const int n_free = *p.n_free;
  const int same = RELEASE ? p.shared / p.page : 0;
  auto pages_of = [&](int n) { return (n + p.page - 1) / p.page; };  // (n < 2^30, a page at most 2^12)
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
  // in place: all blocks have read lengths, counts and the stack's size once they are past the barrier, and their shares
  // below go by shared memory, page tables and the stack alone
  if (blocks > 1) tc::cluster_sync();
  if (rank == 0) {
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
  }
  const int lane = tid & 31, warp = rank * kWarps + (tid >> 5), warps = blocks * kWarps;
  // pages that come or go: a warp takes a run of them
  if (!bad && all_pages > 0) {
    const int n = (int)all_pages, run = ((n + warps - 1) / warps + 31) / 32 * 32;
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
  if (RELEASE) return;
  // rows: a warp takes a run of them, a lane four at a time (their page numbers are on the way together)
  const int64_t run = ((p.n_tokens + warps - 1) / warps + 31) / 32 * 32, first = (int64_t)warp * run, end = min(first + run, p.n_tokens);
  int b = -1;
  for (int64_t i0 = first + lane; i0 < end; i0 += 128) {
    int pos[4], id[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int64_t i = i0 + 32 * u;
      pos[u] = 0, id[u] = -1;
      if (bad || i >= min(end, all_rows)) continue;
      b = b < 0 ? owner(row_s, p.n_seqs, (int)i) : walk(row_s, p.n_seqs, (int)i, b);
      pos[u] = len_s[b] + (int)i - row_s[b];
      const int entry = pos[u] / p.page, mine = pages_of(len_s[b]);
      // a page of this call comes from the stack: its entry may not be written yet
      id[u] = entry < mine ? p.pages[(int64_t)b * p.max_pages + entry] : p.free_pages[n_free - 1 - page_s[b] - (entry - mine)];
      if (id[u] < 0 || id[u] >= p.n_pages) report(p.status, JAB_ERR_INVALID_ARG), id[u] = -1;
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int64_t i = i0 + 32 * u;
      if (i >= end) continue;
      p.positions[i] = pos[u];
      p.slots[i] = id[u] < 0 ? -1 : (int64_t)id[u] * p.page + pos[u] % p.page;
    }
  }
}

template <bool RELEASE>
cudaError_t launch(const KvPlanArgs& a, cudaStream_t st) {
  PlanParams p{};
  p.n_seqs = a.n_seqs, p.page = a.page, p.max_pages = a.max_pages, p.free_capacity = a.free_capacity, p.shared = a.shared;
  p.n_pages = a.n_pages, p.n_tokens = a.n_tokens;
  p.lens = a.lens, p.counts = a.counts, p.n_free = a.n_free;
  p.pages = a.pages, p.free_pages = a.free_pages, p.new_lens = a.new_lens, p.new_free = a.new_free;
  p.q_start = a.q_start, p.positions = a.positions, p.slots = a.slots;
  p.status = a.status;
  auto kern = kv_plan_kernel<RELEASE>;
  static SetUp ready;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  e = ready.once(dev, [&] { return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, 3 * kMostSeqs * 4); });
  if (e != cudaSuccess) return e;
  const int64_t share = RELEASE ? (int64_t)a.n_seqs * 8 : a.n_tokens;
  int blocks = 1;
  while (blocks < kMostBlocks && share > (int64_t)blocks * kRowsPerBlock) blocks *= 2;
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute at[2];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  at[1].id = cudaLaunchAttributeClusterDimension;
  at[1].val.clusterDim.x = blocks;
  at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
  cfg.gridDim = dim3(blocks);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = (size_t)3 * a.n_seqs * 4;
  cfg.stream = st;
  cfg.attrs = at;
  cfg.numAttrs = blocks > 1 ? 2 : 1;
  e = cudaLaunchKernelEx(&cfg, kern, p);
  if (e != cudaSuccess) cudaGetLastError();
  return e;
}

}  // namespace

cudaError_t launch_kv_plan(const KvPlanArgs& a, cudaStream_t st) { return launch<false>(a, st); }
cudaError_t launch_kv_release(const KvPlanArgs& a, cudaStream_t st) { return launch<true>(a, st); }

}  // namespace jab
