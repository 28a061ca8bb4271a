// Shared by the kernels of attention over the quantised cache: arguments, the list of work and how it is cut.
//
// The work of a launch is a list of key tiles in the order (KV head, entry, row tile, key tile). An entry is a
// sequence's queries over the keys of its own, or all queries over the keys that all sequences share; rows are
// (token, query head of the KV head's group) pairs, R of them a tile. Worker c (a warp or a block) takes the tiles [c
// per, (c + 1) per), whatever the lengths: the workers are all resident and finish together. An item (row tile of an entry)
// that is cut, or whose rows have keys in another entry too, leaves its part (maximum, sum, unscaled output) in a
// slot of the workspace for the joining kernel. Every block makes the plan for itself from the lengths on
// the device.
#pragma once

#include "common.cuh"
#include "serve.h"

namespace jab {
namespace kv {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

enum { kTotal = 0, kItems = 1, kPer = 2, kLo = 3, kHi = 4, kLoMax = 5, kHiMin = 6, kPlanHead = 8 };

// One launch's list: which entries it has, and where its plan and parts are.
struct List {
  bool all;                // the shared keys' entry is on it
  int min_rows, max_rows;  // sequences of that many rows are on it
  int32_t* plan;           // kPlanHead scalars
  int4* items;             // [max_items] of a KV head: first token, row tile * 256 + rows, first key tile, key tiles
  int max_items;
  float2* part_ml;         // [n_slots, R]: maximum, sum
  float* part_o;           // [n_slots, R, head_dim]
  int n_slots;
  int used;                // whether the list is run
};

struct AttnParams {
  const uint8_t *k_codes, *v_codes;
  const float *k_scales, *v_scales;
  int n_kv, G, n_pages, max_pages, page;
  int copy_keys;  // keys that are sure to lie in one page, from any multiple of it on: gcd(page, 128)
  FastDiv by_page, by_g;
  const void* q;
  int64_t ldq;
  const int32_t *q_start, *pages, *lens;
  int n_seqs, n_tokens, shared, window;
  float scale_log2;
  void* out;
  int64_t ldo;
  float* lse;
  List list;
  bool behind;  // the launch by keys comes before this one in the call
  int* status;
};

// Elements of Q, O and the log-sum-exps, and of a list's parts, for the checked build.
__device__ __forceinline__ int64_t rows_extent(const AttnParams& p, int64_t pitch, int dh) {
  return (int64_t)(p.n_tokens - 1) * pitch + (int64_t)p.n_kv * p.G * dh;
}
__device__ __forceinline__ bool out_fits(const AttnParams& p, int64_t last, int dh) { return in_bounds(last, rows_extent(p, p.ldo, dh), p.status); }
__device__ __forceinline__ bool lse_fits(const AttnParams& p, int64_t at) { return in_bounds(at, (int64_t)p.n_tokens * p.n_kv * p.G, p.status); }
__device__ __forceinline__ bool part_fits(const AttnParams& p, int64_t last, int rows, int dh) {
  return in_bounds(last, (int64_t)p.list.n_slots * rows * dh, p.status);
}

struct Entry {
  int tok0, nq, len, kbeg;
  bool all;
};

__device__ __forceinline__ Entry sequence(const AttnParams& p, int b) {
  Entry en;
  en.all = false;
  const int s0 = __ldg(p.q_start + b), s1 = __ldg(p.q_start + b + 1);
  en.tok0 = min(max(s0, 0), p.n_tokens);
  en.nq = min(max(s1, en.tok0), p.n_tokens) - en.tok0;
  const int64_t room = min((int64_t)p.max_pages * p.page, (int64_t)INT32_MAX);
  const int len = __ldg(p.lens + b);
  en.len = (int)min((int64_t)max(len, 0), room);
  en.kbeg = p.shared;
  if (s0 != en.tok0 || s1 != en.tok0 + en.nq || len != en.len) report(p.status, JAB_ERR_INVALID_ARG);
  return en;
}

__device__ __forceinline__ int entries(const AttnParams& p) { return p.n_seqs + (p.list.all ? 1 : 0); }

// Entry e of the list; a sequence that is not on it has no rows.
__device__ __forceinline__ Entry entry_of(const AttnParams& p, int e) {
  if (p.list.all && e-- == 0) {
    Entry en;
    en.all = true;
    en.tok0 = 0, en.nq = p.n_tokens, en.len = p.shared, en.kbeg = 0;
    return en;
  }
  Entry en = sequence(p, e);
  const int rows = en.nq * p.G;
  if (rows < p.list.min_rows || rows > p.list.max_rows) en.nq = 0;
  return en;
}

// First key tile (KT keys each) and number of key tiles of row tile rt (at least one: an item that sees
// nothing still has its zeros to write).
template <int R, int KT>
__device__ __forceinline__ void key_tiles(const AttnParams& p, const Entry& en, int rt, const int* head, int& t0, int& n) {
  int lo, hi;
  if (en.all) {
    lo = head[kLo], hi = head[kHi];
  } else {
    const int i0 = p.by_g.quot(rt * R), i1 = p.by_g.quot(min((rt + 1) * R, en.nq * p.G) - 1);
    const int first = en.len - en.nq + 1;
    hi = first + i1;
    lo = max(p.window > 0 ? first + i0 - p.window : 0, en.kbeg);
  }
  t0 = max(lo, 0) / KT;
  n = hi > lo ? max((hi + KT - 1) / KT - t0, 1) : 1;
}

// Keys that every row of [r0, r1) of the entry sees: those in [lo, hi).
__device__ __forceinline__ void seen_by_all(const AttnParams& p, const Entry& en, int r0, int r1, const int* head, int& lo, int& hi) {
  if (en.all) {
    lo = head[kLoMax], hi = head[kHiMin];
  } else {
    const int first = en.len - en.nq + 1;
    hi = first + p.by_g.quot(r0);
    lo = max(p.window > 0 ? first + p.by_g.quot(max(r1 - 1, r0)) - p.window : 0, en.kbeg);
  }
}

// Keys that a row sees: [lo, hi).
__device__ __forceinline__ void seen_by_row(const AttnParams& p, const Entry& en, int pos, int& lo, int& hi) {
  lo = max(en.kbeg, p.window > 0 ? pos + 1 - p.window : 0);
  hi = min(pos + 1, en.len);
}

// Last e with cum[e] <= y (cum[0] = 0 <= y < cum[E]).
__device__ __forceinline__ int find(const int* cum, int E, int y) {
  int lo = 0, hi = E;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (cum[mid] <= y) lo = mid;
    else hi = mid;
  }
  return lo;
}

// Sequence of a token.
__device__ __forceinline__ int sequence_of(const AttnParams& p, int token) {
  int lo = 0, hi = p.n_seqs;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (__ldg(p.q_start + mid) <= token) lo = mid;
    else hi = mid;
  }
  return lo;
}
__device__ __forceinline__ int position_of(const AttnParams& p, int token) {
  const Entry en = sequence(p, sequence_of(p, token));
  return en.len - en.nq + token - en.tok0;
}

// Key tiles and items of a KV head that a list may have. Counts stop there (and are 32-bit numbers for that: q_start and
// lengths of any kind could bring them past 2^31, with shares of the work that begin before the list or behind it).
constexpr int kMostTiles = 1 << 30, kMostItems = 1 << 23;

// The plan, by all WARPS * 32 threads of a block: cum_t[e], cum_i[e] = key tiles and items of a KV head before entry
// e, head[] = the scalars. A list that is too long is reported and counts as empty.
template <int R, int KT, int WARPS>
__device__ void make_plan(const AttnParams& p, int workers, int* cum_t, int* cum_i, int* head) {
  __shared__ int w_v[4][WARPS];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, E = entries(p);
  if (p.list.all) {  // what the queries see of the shared keys: any of them, and all of them
    int v[4] = {p.shared, 0, 0, p.shared};
    for (int b = tid; b < p.n_seqs; b += 32 * WARPS) {
      const Entry en = sequence(p, b);
      if (en.nq > 0) {
        const int first = en.len - en.nq + 1;
        v[0] = min(v[0], p.window > 0 ? max(first - p.window, 0) : 0);
        v[1] = max(v[1], min(en.len, p.shared));
        v[2] = max(v[2], p.window > 0 ? en.len - p.window : 0);
        v[3] = min(v[3], first);
      }
    }
    v[0] = __reduce_min_sync(0xffffffffu, v[0]);
    v[1] = __reduce_max_sync(0xffffffffu, v[1]);
    v[2] = __reduce_max_sync(0xffffffffu, v[2]);
    v[3] = __reduce_min_sync(0xffffffffu, v[3]);
    if (lane == 0)
      for (int i = 0; i < 4; ++i) w_v[i][warp] = v[i];
    __syncthreads();
    if (tid == 0) {
      for (int w = 1; w < WARPS; ++w) {
        v[0] = min(v[0], w_v[0][w]), v[1] = max(v[1], w_v[1][w]);
        v[2] = max(v[2], w_v[2][w]), v[3] = min(v[3], w_v[3][w]);
      }
      head[kLo] = v[0], head[kHi] = v[1], head[kLoMax] = v[2], head[kHiMin] = v[3];
    }
    __syncthreads();
  } else if (tid == 0) {
    head[kLo] = head[kHi] = head[kLoMax] = head[kHiMin] = 0;
  }
  const int run = (E + 32 * WARPS - 1) / (32 * WARPS);
  const int e0 = min(tid * run, E), e1 = min(e0 + run, E);
  int st = 0, si = 0;
#pragma unroll 1
  for (int pass = 0; pass < 2; ++pass) {
    int at = 0, ai = 0;
    if (pass == 1) {  // exclusive prefix over the threads
      int t = st, i = si;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int ut = __shfl_up_sync(0xffffffffu, t, o), ui = __shfl_up_sync(0xffffffffu, i, o);
        if (lane >= o) t = min(t + ut, kMostTiles), i = min(i + ui, kMostItems);
      }
      if (lane == 31) w_v[0][warp] = t, w_v[1][warp] = i;
      __syncthreads();
      at = t - st, ai = i - si;
      for (int w = 0; w < warp; ++w) at = min(at + w_v[0][w], kMostTiles), ai = min(ai + w_v[1][w], kMostItems);
    }
    for (int e = e0; e < e1; ++e) {
      const Entry en = entry_of(p, e);
      const int nrt = (en.nq * p.G + R - 1) / R;
      if (pass == 1) cum_t[e] = at, cum_i[e] = ai;
      int sum = 0, t0, n;
      if (en.all) {
        key_tiles<R, KT>(p, en, 0, head, t0, n);
        sum = (int)min((int64_t)n * nrt, (int64_t)kMostTiles);
      } else if (nrt < kMostItems) {
        for (int rt = 0; rt < nrt; ++rt) {
          key_tiles<R, KT>(p, en, rt, head, t0, n);
          sum = min(sum + n, kMostTiles);
        }
      }
      at = min(at + sum, kMostTiles), ai = min(ai + nrt, kMostItems);
    }
    if (pass == 0) st = at, si = ai;
  }
  if (tid == 0) {
    int t = 0, i = 0;
    for (int w = 0; w < WARPS; ++w) t = min(t + w_v[0][w], kMostTiles), i = min(i + w_v[1][w], kMostItems);
    int64_t per = ((int64_t)t * p.n_kv + workers - 1) / workers;
    if (t >= kMostTiles || i >= kMostItems || per > INT32_MAX) {
      t = i = per = 0;
      if (blockIdx.x == 0) report(p.status, JAB_ERR_INVALID_ARG);
    }
    cum_t[E] = t, cum_i[E] = i;
    head[kTotal] = t, head[kItems] = i, head[kPer] = (int)per;
  }
  __syncthreads();
  if (blockIdx.x != 0) return;
  // rows that no sequence owns would stay as they are
  if (tid == 0 && (__ldg(p.q_start) != 0 || __ldg(p.q_start + p.n_seqs) != p.n_tokens)) report(p.status, JAB_ERR_INVALID_ARG);
  // for the joining kernel: the scalars, and every item
  for (int i = tid; i < kPlanHead; i += 32 * WARPS) p.list.plan[i] = head[i];
  if (head[kItems] == 0) return;
  for (int e = tid; e < E; e += 32 * WARPS) {
    const Entry en = entry_of(p, e);
    int at = cum_t[e], i = cum_i[e], t0, n;
    for (int rt = 0; i < cum_i[e + 1]; ++rt, ++i, at += n) {
      key_tiles<R, KT>(p, en, rt, head, t0, n);
      if (i < p.list.max_items)
        p.list.items[i] = make_int4(en.tok0, rt * 256 + min(R, en.nq * p.G - rt * R), at, n);
      else
        report(p.status, JAB_ERR_INVALID_ARG);
    }
  }
}

// The item that tile x of the list is in.
struct Item {
  Entry en;
  int h, e, rt;     // KV head, entry, row tile
  int t0, n;        // its first key tile and their number
  int s0, s1;       // the part of them, counted from t0, that is this worker's
  int rows;         // rows of the tile in use
};
template <int R, int KT>
__device__ __forceinline__ Item item_at(const AttnParams& p, const int* cum_t, const int* head, int64_t x, int64_t x1) {
  Item it;
  const int total = head[kTotal];
  it.h = (int)(x / total);
  const int y = (int)(x - (int64_t)it.h * total);
  it.e = find(cum_t, entries(p), y);
  it.en = entry_of(p, it.e);
  int base = cum_t[it.e];
  it.rt = 0;
  key_tiles<R, KT>(p, it.en, 0, head, it.t0, it.n);
  if (it.en.all) {
    it.rt = (y - base) / it.n;
    base += it.rt * it.n;
  } else {
    while (y >= base + it.n) {
      base += it.n;
      key_tiles<R, KT>(p, it.en, ++it.rt, head, it.t0, it.n);
    }
  }
  it.s0 = y - base;
  it.s1 = (int)min((int64_t)it.n, it.s0 + (x1 - x));
  it.rows = min(R, it.en.nq * p.G - it.rt * R);
  return it;
}

// Where a part goes. With shared keys every item leaves a part (worker + item counts up along the list); without,
// only the first and the last of a worker can be cut.
__device__ __forceinline__ int64_t slot_of(const AttnParams& p, int worker, int item, bool first) {
  return p.shared > 0 ? (int64_t)worker + item : 2 * (int64_t)worker + (first ? 0 : 1);
}

// log2 of the least V scale that the running maxima know: one below it (a row of zeros) counts as this. Such a key's
// weight is small whatever its score is, its 2^(s - m) is not: like this, that is at most 2^104 when the maximum follows
// from 2^8 on, and the sums of 2^23 of them are finite.
// A scale of NaN (or infinity) counts as 1: the row's output is NaN, its log-sum-exp stays right.
constexpr float kLeastLog2 = -90.f;

// The maxima are held 2^6 lower than they are, in both kernels: a row's largest weight is then 2^6 and more as it goes
// into the products (2^15 at most, where the maximum follows from 2^8 on), and what fp16 cannot hold of a small one,
// 2^-25, is 2^-31 of that. (Held at 1, a flat tail of weights 2^-26 of one key's was lost from the outputs, though not
// from the sums that they are divided by: 2^-10 of the result for 65536 keys.)
constexpr float kHeadroom = 6.f;

// 2^(a - b) with 2^(-inf - -inf) = 0.
__device__ __forceinline__ float shift2(float a, float b) { return a == -INFINITY ? 0.f : exp2f(a - b); }

template <class T>
__device__ __forceinline__ void store_out(T* p, float v);
template <>
__device__ __forceinline__ void store_out<half_t>(half_t* p, float v) { *p = __float2half_rn(v); }
template <>
__device__ __forceinline__ void store_out<bf16_t>(bf16_t* p, float v) { *p = __float2bfloat16_rn(v); }

// Power of two that brings a bf16 row whose largest magnitude has the bits `big` to [2^14, 2^15), the last octave but
// one of fp16, and its inverse. The row's elements from 2^-31 of the largest on are then exact in fp16 (their last of
// eight bits is at 2^-24 or above), the others within 2^-39 of it. Both powers are normal numbers; the largest bf16
// exponent comes to the last octave.
__device__ __forceinline__ void row_power(uint32_t big, float& by, float& back) {
  const int e = min(max((int)(big >> 23), 15), 253);
  by = __uint_as_float((uint32_t)(268 - e) << 23);    // 2^(141 - e)
  back = __uint_as_float((uint32_t)(e - 14) << 23);   // 2^(e - 141)
}

// Tile kernel (kv_attn_tile.cu): 128 rows x 128 keys on the tensor cores.
constexpr int kTileRows = 128, kTileKeys = 128;
cudaError_t launch_tiles(const AttnParams& p, jab_dtype type, int dh, int bits, int64_t est_tiles, int sms, cudaStream_t st);

}  // namespace kv
}  // namespace jab
