// Attention over the quantised paged cache for many rows that see the same keys (chunks of a prompt, a prefix that
// all sequences share): 128 rows x 128 keys at a time on the tensor cores, by the formulas of kv_attn.cu.
//
// The codes of a key tile come as the bytes that they are, by bulk copies of the keys that share a page, and become
// fp16 in shared memory once per tile; the scales stay outside of the products as they do there. (Loaded straight to
// the converters' registers they would pass shared memory once less, but 128 threads have too few bytes in flight:
// 2 x 512 queries behind 5000 keys took 292 us, by bulk copies 167 at that time.)
// Both products are M128 N128 with their A operand in tensor memory:
//   S = Q K^T   A = Q (fp16, written to tensor memory row by row), B = K as converted (K-major)
//   O += P V    A = P (fp16 weights, written by the softmax), B = V as converted (MN-major: the same layout)
// P is its fp16 value and what that leaves over (2^-22 of a weight in all), in two products, as in the kernel by
// keys: rounded once, a weight would be 2^-11 off, and what a token gets would hang on which of the two kernels its
// batch brings it to.
//   warp 0        bulk copies of codes and scales, rings of KST and VST tiles
//   warp 1        tensor memory owner; issues S, a tile ahead of P V;   warp 2  issues P V
//   warp 3        finds the block's items, ahead of all, and leaves them in a ring (each warp for itself: 1 to 2 us an item)
//   warps 4..11   softmax: 16 rows a warp, four threads a row (16x256b shape); at an item's end the output
//   warps 12..15  converters of K, a tile ahead; of Q at an item's start, and of the keys' scales
//   warps 16..19  converters of V
// Bound: no unit, but the latency of the softmax: 2800 of the 3500 clocks that a 128 x 128 tile takes (with clock stamps),
// the issue slots half used (2 x 512 queries, 4100 to 6000 keys, window 4096, 32 heads of 128: 122 us and 28 to join,
// tensor pipe 32 % busy). With one part of a weight where no mask cuts, the call took as long: the second product runs
// beside the next softmax. Where items are short, the first tile of each, which looks for the maximum first, its Q and its
// output are what counts: 12 prompts of 482 tokens over their own keys take 272 us, one of 2048 207, where Q, O and the
// products need 16 and 18.
#include <algorithm>
#include <type_traits>

#include "kv_attn.cuh"
#include "per_device.h"
#include "tc.cuh"

namespace jab {
namespace kv {
namespace {

constexpr int R = kTileRows, KT = kTileKeys, THREADS = 640, SCB = 3, KST = 2, VST = 2, IST = 4;

template <int DH, int BITS>
struct Layout {
  static constexpr int CHUNK = 128 * 128;              // 128 keys x 64 dimensions of fp16, 128-byte swizzle
  static constexpr int TILE = KT * DH * 2;             // K or V in fp16
  static constexpr int RAW = KT * DH * BITS / 8;       // K or V as codes
  static constexpr int K_STAGE = RAW + 2 * KT * 4;     // K and the scales of both
  static constexpr int K_OFF = 0, V_OFF = 2 * TILE, RK_OFF = 4 * TILE, RV_OFF = RK_OFF + KST * K_STAGE;
  static constexpr int SC_OFF = RV_OFF + VST * RAW;                         // per tile: K scale * log2 e * c, V scale, its log2 less the headroom
  static constexpr int ROW_OFF = SC_OFF + SCB * 3 * KT * 4;       // per item: lo, hi, power of two of Q
  static constexpr int BAR_OFF = ROW_OFF + 2 * 3 * R * 4;
  static constexpr int ITEM_OFF = BAR_OFF + 512;
  static constexpr int USED = ITEM_OFF + IST * 64;
  // Two S of 128 columns. P takes their place, 64 keys at a time: 32 columns of fp16 pairs, 32 of what they leave over.
  static constexpr uint32_t S_COL = 0, O_COL = 256, Q_COL = 384;
};

struct Bars {
  uint64_t rk_full[KST], rk_empty[KST], rv_full[VST], rv_empty[VST], k_full[2], k_empty[2], sc_full[SCB], sc_empty[SCB], v_full[2], v_empty[2];
  uint64_t item_full[IST], item_empty[IST], q_full[2], q_empty, rows_empty[2], s_full[2], s_empty[2], p_full[2], pv_done[2], o_full, o_empty, drain[2];
  uint32_t tmem_base;
  int abort;
};
static_assert(sizeof(Bars) <= 512, "barrier block");

// An item as warp 3 leaves it.
struct Record {
  int h, e, rt, t0, n, s0, s1, rows, tok0, nq, len, kbeg, all, lo, hi, part;  // lo, hi: keys that all rows see; part: item of the list
};
constexpr int kReaders = 3 + 8 + 4;  // warps that read it

__device__ __forceinline__ void drain_wait(uint64_t* bar, uint32_t parity) {
  const uint64_t t0 = tc::globaltimer();
  while (!tc::mbar_test(bar, parity))
    if (tc::globaltimer() - t0 > tc::kWaitLimitNs) break;
}

template <int N>
__device__ __forceinline__ void more_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N>
__device__ __forceinline__ void fewer_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }

__device__ __forceinline__ uint32_t biased_h2(uint32_t u, uint32_t bias2) {
  const __half2 r = __hsub2(*reinterpret_cast<const __half2*>(&u), *reinterpret_cast<const __half2*>(&bias2));
  return *reinterpret_cast<const uint32_t*>(&r);
}

// 8 codes (8 or 4 bytes) as fp16, in their order.
__device__ __forceinline__ uint4 eight_codes(uint2 w) {
  constexpr uint32_t k = 0x64806480u;  // 1152
  uint4 r;
  r.x = biased_h2(__byte_perm(w.x, 0x64646464u, 0x4140), k);
  r.y = biased_h2(__byte_perm(w.x, 0x64646464u, 0x4342), k);
  r.z = biased_h2(__byte_perm(w.y, 0x64646464u, 0x4140), k);
  r.w = biased_h2(__byte_perm(w.y, 0x64646464u, 0x4342), k);
  return r;
}
__device__ __forceinline__ uint4 eight_codes(uint32_t w) {
  constexpr uint32_t k = 0x64086408u;  // 1032
  const uint32_t even = w & 0x0f0f0f0fu, odd = (w >> 4) & 0x0f0f0f0fu;
  const uint32_t a = __byte_perm(even, odd, 0x5140), b = __byte_perm(even, odd, 0x7362);
  uint4 r;
  r.x = biased_h2(__byte_perm(a, 0x64646464u, 0x4140), k);
  r.y = biased_h2(__byte_perm(a, 0x64646464u, 0x4342), k);
  r.z = biased_h2(__byte_perm(b, 0x64646464u, 0x4140), k);
  r.w = biased_h2(__byte_perm(b, 0x64646464u, 0x4342), k);
  return r;
}

// A tile of codes to fp16 in the swizzled layout, by 128 threads: consecutive threads take consecutive eights of a
// row, so that reads and 16-byte writes are free of bank conflicts. (A batch is read before any of it is written: the
// compiler cannot know that the two do not overlap.)
template <int DH, int BITS>
__device__ __forceinline__ void convert_tile(const uint8_t* raw, uint8_t* dst, int tid) {
  using Word = std::conditional_t<BITS == 8, uint2, uint32_t>;
  constexpr int N = KT * DH / 8 / 128, PER_ROW = DH / 8;
#pragma unroll 1
  for (int i0 = 0; i0 < N; i0 += 4) {
    Word w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = reinterpret_cast<const Word*>(raw)[tid + (i0 + i) * 128];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int key = (tid + (i0 + i) * 128) / PER_ROW, c = tid % PER_ROW;
      *reinterpret_cast<uint4*>(dst + (c >> 3) * (128 * 128) + key * 128 + (((c & 7) ^ (key & 7)) << 4)) = eight_codes(w[i]);
    }
  }
}

// 32 scores of a thread: rows c = 0, 1 of the warp's pairs, columns c0 + 8n + e (n < 8, e < 2) of the tile as the 16x256b
// shape gives them, c0 = 2 (lane % 4) + 64 b. sc: the tile's K scales from column c0 on; V scales and their logarithms
// are KT and 2 KT floats further. y = score - ref.
template <class T>
__device__ __forceinline__ float2 score(const uint32_t* e, float2 ks, float fac, float ref) {
  float2 a = make_float2(__uint_as_float(e[0]), __uint_as_float(e[1]));
  if constexpr (std::is_same<T, bf16_t>::value) a = tc::mul2(a, make_float2(fac, fac));
  return tc::fma2(a, ks, make_float2(-ref, -ref));
}

// Rows c = 0, 1 of DH accumulator columns times f[c].
template <int DH>
__device__ __forceinline__ void scale_rows(uint32_t taddr, const float (&f)[2]) {
#pragma unroll 1
  for (int b = 0; b < DH / 32; ++b) {
    uint32_t o[16];
    tc::tmem_ld_16x256b_x4(taddr + 32 * b, o);
    tc::tmem_ld_wait();
#pragma unroll
    for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * f[(k >> 1) & 1]);
    tc::tmem_st_16x256b_x4(taddr + 32 * b, o);
  }
  tc::tmem_st_wait();
}

// A pair of weights as fp16, and what that leaves over.
__device__ __forceinline__ void two_parts(float2 w, uint32_t& h, uint32_t& r) {
  h = tc::pack_half2(w.x, w.y);
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
  r = tc::pack_half2(w.x - f.x, w.y - f.y);
}

// Weights of keys that no mask hides, in the scores' place: v[4n + 2c] becomes the pair in fp16, v[4n + 2c + 1] what
// that leaves over; l gets the row sums of 2^y, `big` the largest weight of either half of the pairs. As long as none
// passes 2^15 and no sum 2^112 the reference may stay, and neither the maximum nor the V scales' logarithms are
// needed. (The sums: a key whose values are zero has no weight, however far its score is ahead. Once the reference has
// moved its 2^y is at most 2^96, and a sum has room for 2^16 more of them.)
template <class T>
__device__ __forceinline__ void plain_weights(uint32_t (&v)[32], const float* sc, const float (&ref)[2], const float (&fac)[2], float2 (&l)[2], uint32_t& big) {
  big = 0;
#pragma unroll
  for (int n = 0; n < 8; ++n) {
    const float2 ks = *reinterpret_cast<const float2*>(sc + 8 * n), vs = *reinterpret_cast<const float2*>(sc + KT + 8 * n);
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      uint32_t* e = v + 4 * n + 2 * c;
      const float2 y = score<T>(e, ks, fac[c], ref[c]);
      const float2 ex = make_float2(tc::fast_exp2(y.x), tc::fast_exp2(y.y));
      l[c] = tc::add2(l[c], ex);
      two_parts(tc::mul2(ex, vs), e[0], e[1]);
      big = __vmaxu2(big, e[0]);
    }
  }
}

__device__ __forceinline__ bool sums_fit(const float2 (&l)[2]) { return fmaxf(fmaxf(l[0].x, l[0].y), fmaxf(l[1].x, l[1].y)) < 5.192297e33f; }

// Stores 64 keys' weights as plain_weights and masked_weights leave them.
__device__ __forceinline__ void store_weights(uint32_t taddr, const uint32_t (&v)[32]) {
  uint32_t w[32];
#pragma unroll
  for (int k = 0; k < 16; ++k) w[k] = v[2 * k], w[16 + k] = v[2 * k + 1];
  tc::tmem_st_16x128b_x16(taddr, w);
}

__device__ __forceinline__ uint32_t pair_as(float a, float b, half_t) { return tc::pack_half2(a, b); }
__device__ __forceinline__ uint32_t pair_as(float a, float b, bf16_t) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// Whether the row with bounds [lo, hi) sees keys k, k + 1.
struct Sees {
  bool x, y;
  __device__ __forceinline__ Sees(int k, int lo, int hi) : x(k >= lo && k < hi), y(k + 1 >= lo && k + 1 < hi) {}
};

// The rows' largest score + log2 of the key's V scale (less the headroom), with masks. (A hidden key's scales may be anything.)
template <class T>
__device__ __forceinline__ void masked_top(const uint32_t (&v)[32], const float* sc, const float (&fac)[2], const int (&lo)[2], const int (&hi)[2], int k0,
                                           float (&top)[2]) {
#pragma unroll
  for (int n = 0; n < 8; ++n) {
    const float2 ks = *reinterpret_cast<const float2*>(sc + 8 * n), lv = *reinterpret_cast<const float2*>(sc + 2 * KT + 8 * n);
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const float2 u = tc::add2(score<T>(v + 4 * n + 2 * c, ks, fac[c], 0.f), lv);
      const Sees see(k0 + 8 * n, lo[c], hi[c]);
      top[c] = tc::fmax3(top[c], see.x ? u.x : -INFINITY, see.y ? u.y : -INFINITY);
    }
  }
}
// The masked tile's weights in place: v[4n + 2c] becomes the pair in fp16, v[4n + 2c + 1] what that leaves over.
template <class T>
__device__ __forceinline__ void masked_weights(uint32_t (&v)[32], const float* sc, const float (&ref)[2], const float (&fac)[2], const int (&lo)[2],
                                               const int (&hi)[2], int k0, float2 (&l)[2]) {
#pragma unroll
  for (int n = 0; n < 8; ++n) {
    const float2 ks = *reinterpret_cast<const float2*>(sc + 8 * n), vs = *reinterpret_cast<const float2*>(sc + KT + 8 * n);
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      uint32_t* e = v + 4 * n + 2 * c;
      const float2 y = score<T>(e, ks, fac[c], ref[c]);
      const Sees see(k0 + 8 * n, lo[c], hi[c]);
      const float2 ex = make_float2(see.x ? tc::fast_exp2(y.x) : 0.f, see.y ? tc::fast_exp2(y.y) : 0.f);
      l[c] = tc::add2(l[c], ex);
      two_parts(make_float2(see.x ? ex.x * vs.x : 0.f, see.y ? ex.y * vs.y : 0.f), e[0], e[1]);
    }
  }
}

template <class T, int DH, int BITS>
__global__ void __launch_bounds__(THREADS, 1) kv_tile_kernel(const __grid_constant__ AttnParams p) {
  using L = Layout<DH, BITS>;
  extern __shared__ uint8_t smem_raw[];
  __shared__ int head[kPlanHead];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  Bars* bars = reinterpret_cast<Bars*>(smem + L::BAR_OFF);
  const int E = entries(p);
  int* cum_t = reinterpret_cast<int*>(smem + L::USED);
  int* cum_i = cum_t + E + 1;
  const int warp = tc::warp_index(), lane = threadIdx.x & 31;
  volatile int* abort = &bars->abort;
  if (threadIdx.x == 0) {
    for (int s = 0; s < 2; ++s) {
      tc::mbar_init(&bars->k_full[s], 4);
      tc::mbar_init(&bars->k_empty[s], 1);
      tc::mbar_init(&bars->drain[s], 1);
      tc::mbar_init(&bars->q_full[s], 4);
      tc::mbar_init(&bars->rows_empty[s], 8);
      tc::mbar_init(&bars->p_full[s], 8);
      tc::mbar_init(&bars->pv_done[s], 1);
      tc::mbar_init(&bars->v_full[s], 4);
      tc::mbar_init(&bars->v_empty[s], 1);
      tc::mbar_init(&bars->s_full[s], 1);
      tc::mbar_init(&bars->s_empty[s], 1);  // (P V has read the weights that took the scores' place)
    }
    for (int s = 0; s < IST; ++s) {
      tc::mbar_init(&bars->item_full[s], 1);
      tc::mbar_init(&bars->item_empty[s], kReaders);
    }
    for (int s = 0; s < KST; ++s) {
      tc::mbar_init(&bars->rk_full[s], 1);
      tc::mbar_init(&bars->rk_empty[s], 4);
    }
    for (int s = 0; s < VST; ++s) {
      tc::mbar_init(&bars->rv_full[s], 1);
      tc::mbar_init(&bars->rv_empty[s], 4);
    }
    for (int s = 0; s < SCB; ++s) {
      tc::mbar_init(&bars->sc_full[s], 4);
      tc::mbar_init(&bars->sc_empty[s], 8);
    }
    tc::mbar_init(&bars->q_empty, 1);
    tc::mbar_init(&bars->o_full, 1);
    tc::mbar_init(&bars->o_empty, 8);
    bars->abort = 0;
    tc::fence_mbar_init();
  }
  if (warp == 1) {
    tc::tmem_alloc(&bars->tmem_base, 512);
    tc::tmem_relinquish();
  }
  tc::fence_before_sync();
  __syncthreads();
  tc::fence_after_sync();
  const uint32_t tmem = __shfl_sync(0xffffffffu, bars->tmem_base, 0);
  // Behind the launch by keys there is nothing to wait for yet: that one let this one in only when all before it was
  // complete, and neither reads what the other writes. The joining kernel waits for this one's end, which waits below.
  // (64 sequences behind 8192 shared keys: 75 us in all one after the other, 67 like this.)
  if (p.behind)
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  else
    stream_order();
  make_plan<R, KT, THREADS / 32>(p, gridDim.x, cum_t, cum_i, head);
  const int64_t all = (int64_t)head[kTotal] * p.n_kv;
  const int64_t x0 = (int64_t)blockIdx.x * head[kPer], x1 = min(all, x0 + head[kPer]);
  Record* ring = reinterpret_cast<Record*>(smem + L::ITEM_OFF);
  // The block's i-th item, for a warp that reads them all in turn.
  auto take = [&](int i, Record& it) -> bool {
    if (!__all_sync(0xffffffffu, tc::mbar_wait(&bars->item_full[i % IST], (i / IST) & 1, abort, p.status))) return false;
    it = ring[i % IST];
    __syncwarp();
    if (lane == 0) tc::mbar_arrive(&bars->item_empty[i % IST]);
    return true;
  };
  // Every role walks the block's items; j counts key tiles and i items over all of them.
  if (warp < 4) {
    fewer_registers<48>();
    if (warp == 0) {  // ---------------- bulk copies
      int j = 0, i = 0;
      bool ok = true;
      // lane: one of K, its scales, V's scales, V; and a group of keys that lie in one page
      const int kind = lane >> 3, grp = lane & 7, size = p.copy_keys;
      const uint8_t* src = kind == 0   ? p.k_codes
                           : kind == 1 ? reinterpret_cast<const uint8_t*>(p.k_scales)
                           : kind == 2 ? reinterpret_cast<const uint8_t*>(p.v_scales)
                                       : p.v_codes;
      constexpr int ROW = DH * BITS / 8;
      const int row_bytes = kind == 1 || kind == 2 ? 4 : ROW;
      const int off = (kind == 1 ? L::RAW : kind == 2 ? L::RAW + KT * 4 : 0) + grp * size * row_bytes;
      for (int64_t x = x0; x < x1 && ok; ++i) {
        Record it;
        if (!(ok = take(i, it))) break;
        const int32_t* table = p.pages + (it.all ? 0 : (int64_t)(it.e - (p.list.all ? 1 : 0)) * p.max_pages);
        // Cache row of this lane's group of tile s; -1: past the keys (what is in its place is hidden).
        auto row_of = [&](int s) -> int64_t {
          const int key = (it.t0 + s) * KT + grp * size;
          if (grp * size >= KT || key >= it.len || s >= it.s1) return -1;
          const int pg = p.by_page.quot(key);
          int id = __ldg(table + pg);
          if (id < 0 || id >= p.n_pages) {
            report(p.status, JAB_ERR_INVALID_ARG);
            id = 0;
          }
          return ((int64_t)id * p.n_kv + it.h) * p.page + (key - pg * p.page);
        };
        int64_t row = row_of(it.s0);
        for (int s = it.s0; s < it.s1; ++s, ++j) {
          const int ks = j % KST, vs = j % VST;
          const unsigned n = __popc(__ballot_sync(0xffffffffu, row >= 0) & 0xffu) * size;
          ok = __all_sync(0xffffffffu, tc::mbar_wait(&bars->rk_empty[ks], ((j / KST) & 1) ^ 1, abort, p.status));
          if (!ok) break;
          if (lane == 0) tc::mbar_expect_tx(&bars->rk_full[ks], n * (ROW + 8));
          __syncwarp();
          if (kind < 3 && row >= 0)
            tc::bulk_load(smem + L::RK_OFF + ks * L::K_STAGE + off, src + row * row_bytes, size * row_bytes, &bars->rk_full[ks]);
          ok = __all_sync(0xffffffffu, tc::mbar_wait(&bars->rv_empty[vs], ((j / VST) & 1) ^ 1, abort, p.status));
          if (!ok) {
            drain_wait(&bars->rk_full[ks], (j / KST) & 1);
            break;
          }
          if (lane == 0) tc::mbar_expect_tx(&bars->rv_full[vs], n * ROW);
          __syncwarp();
          if (kind == 3 && row >= 0)
            tc::bulk_load(smem + L::RV_OFF + vs * L::RAW + off, src + row * row_bytes, size * row_bytes, &bars->rv_full[vs]);
          row = row_of(s + 1);  // (its page number arrives while the rings are full)
        }
        x += it.s1 - it.s0;
      }
      if (*abort) {  // every copy issued has landed before shared memory goes to another block
        for (int k = max(0, j - KST); k < j; ++k) drain_wait(&bars->rk_full[k % KST], (k / KST) & 1);
        for (int k = max(0, j - VST); k < j; ++k) drain_wait(&bars->rv_full[k % VST], (k / VST) & 1);
      }
    } else if (warp == 1) {  // ---------------- S (the whole warp waits, one thread issues: see the projection's kernel)
      constexpr uint32_t IDESC = tc::idesc_f16(false, R, KT);
      int j = 0, i = 0;
      bool ok = true;
      for (int64_t x = x0; x < x1 && ok; ++i) {
        Record it;
        if (!(ok = take(i, it))) break;
        ok = __all_sync(0xffffffffu, tc::mbar_wait(&bars->q_full[i & 1], (i >> 1) & 1, abort, p.status));
        for (int s = it.s0; s < it.s1 && ok; ++s, ++j) {
          ok = __all_sync(0xffffffffu, tc::mbar_wait(&bars->k_full[j & 1], (j >> 1) & 1, abort, p.status) &&
                                           tc::mbar_wait(&bars->s_empty[j & 1], ((j >> 1) & 1) ^ 1, abort, p.status));
          if (ok && tc::elect_one()) {
            tc::fence_after_sync();
            const uint64_t kd = tc::sdesc_kmajor_sw128(tc::smem_u32(smem + L::K_OFF + (j & 1) * L::TILE));
#pragma unroll
            for (int k = 0; k < DH / 16; ++k)
              tc::umma_f16_ts(tmem + L::S_COL + (j & 1) * KT, tmem + L::Q_COL + k * 8, tc::sdesc_advance(kd, (k >> 2) * L::CHUNK + (k & 3) * 32), IDESC,
                              k > 0 ? 1u : 0u);
            tc::umma_commit(&bars->s_full[j & 1]);
            tc::umma_commit(&bars->k_empty[j & 1]);
            if (s + 1 == it.s1) tc::umma_commit(&bars->q_empty);
          }
          __syncwarp();
        }
        x += it.s1 - it.s0;
      }
      if (tc::elect_one()) {
        tc::umma_commit(&bars->drain[0]);
        drain_wait(&bars->drain[0], 0);
      }
    } else if (warp == 2) {  // ---------------- P V
      constexpr uint32_t IDESC = tc::idesc_f16(false, R, DH) | (1u << 16);  // B MN-major
      int j = 0, i = 0;
      bool ok = true;
      for (int64_t x = x0; x < x1 && ok; ++i) {
        Record it;
        if (!(ok = take(i, it))) break;
        ok = __all_sync(0xffffffffu, tc::mbar_wait(&bars->o_empty, (i & 1) ^ 1, abort, p.status));
        for (int s = it.s0; s < it.s1 && ok; ++s, ++j) {
          ok = __all_sync(0xffffffffu, tc::mbar_wait(&bars->v_full[j & 1], (j >> 1) & 1, abort, p.status) &&
                                           tc::mbar_wait(&bars->p_full[j & 1], (j >> 1) & 1, abort, p.status));
          if (ok && tc::elect_one()) {
            tc::fence_after_sync();
            const uint64_t vd = tc::sdesc_mnmajor_sw128(tc::smem_u32(smem + L::V_OFF + (j & 1) * L::TILE), L::CHUNK, 1024);
#pragma unroll
            for (int part = 0; part < 2; ++part)
#pragma unroll
              for (int k = 0; k < KT / 16; ++k)
                tc::umma_f16_ts(tmem + L::O_COL, tmem + L::S_COL + (j & 1) * KT + (k >> 2) * 64 + part * 32 + (k & 3) * 8, tc::sdesc_advance(vd, k * 16 * 128),
                                IDESC, s > it.s0 || part > 0 || k > 0 ? 1u : 0u);
            tc::umma_commit(&bars->pv_done[j & 1]);
            tc::umma_commit(&bars->s_empty[j & 1]);
            tc::umma_commit(&bars->v_empty[j & 1]);
            if (s + 1 == it.s1) tc::umma_commit(&bars->o_full);
          }
          __syncwarp();
        }
        x += it.s1 - it.s0;
      }
      if (tc::elect_one()) {
        tc::umma_commit(&bars->drain[1]);
        drain_wait(&bars->drain[1], 0);
      }
    }
    else if (warp == 3) {  // ---------------- items
      int i = 0;
      for (int64_t x = x0; x < x1; ++i) {
        const Item it = item_at<R, KT>(p, cum_t, head, x, x1);
        Record rec{it.h, it.e, it.rt, it.t0, it.n, it.s0, it.s1, it.rows, it.en.tok0, it.en.nq, it.en.len, it.en.kbeg, it.en.all, 0, 0, 0};
        seen_by_all(p, it.en, it.rt * R, it.rt * R + it.rows, head, rec.lo, rec.hi);
        rec.part = it.h * head[kItems] + cum_i[it.e] + it.rt;
        if (!__all_sync(0xffffffffu, tc::mbar_wait(&bars->item_empty[i % IST], ((i / IST) & 1) ^ 1, abort, p.status))) break;
        if (lane == 0) {
          ring[i % IST] = rec;
          tc::mbar_arrive(&bars->item_full[i % IST]);
        }
        __syncwarp();
        x += it.s1 - it.s0;
      }
    }
  } else if (warp < 12) {  // ---------------- softmax
    more_registers<128>();
    const int quarter = warp & 3, g = lane >> 2, q4 = lane & 3;
    const int r0 = 32 * quarter + 16 * ((warp - 4) >> 2);  // the warp's first row
    const uint32_t tw = tmem + ((uint32_t)r0 << 16);
    int j = 0, i = 0;
    bool ok = true;
    for (int64_t x = x0; x < x1 && ok; ++i) {
      Record it;
      if (!(ok = take(i, it))) break;
      float m[2] = {-INFINITY, -INFINITY};
      float2 l[2] = {};
      if (!(ok = tc::mbar_wait(&bars->q_full[i & 1], (i >> 1) & 1, abort, p.status))) break;  // (the rows' bounds are written before it)
      const int* rows_lo = reinterpret_cast<const int*>(smem + L::ROW_OFF + (i & 1) * 3 * R * 4);
      int lo[2], hi[2];
      float fac[2];
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        lo[c] = rows_lo[r0 + g + 8 * c], hi[c] = rows_lo[R + r0 + g + 8 * c];
        fac[c] = __int_as_float(rows_lo[2 * R + r0 + g + 8 * c]);
      }
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(&bars->rows_empty[i & 1]);
      for (int s = it.s0; s < it.s1; ++s, ++j) {
        const float* sc = reinterpret_cast<const float*>(smem + L::SC_OFF + (j % SCB) * 3 * KT * 4) + 2 * q4;
        if (!(ok = tc::mbar_wait(&bars->sc_full[j % SCB], (j / SCB) & 1, abort, p.status) &&
                   tc::mbar_wait(&bars->s_full[j & 1], (j >> 1) & 1, abort, p.status)))
          break;
        tc::fence_after_sync();
        const int key0 = (it.t0 + s) * KT;
        const bool masked = key0 < it.lo || key0 + KT > it.hi;
        const uint32_t ts = tw + L::S_COL + (j & 1) * KT;
        // P V of the tile before is done: O may be rescaled
        auto before_o = [&]() -> bool {
          if (j > 0 && !tc::mbar_wait(&bars->pv_done[(j - 1) & 1], ((j - 1) >> 1) & 1, abort, p.status)) return false;
          tc::fence_after_sync();
          __syncwarp();
          return true;
        };
        // Weights take the place of the scores that have been read, 64 keys at a time (a loop, not two copies: what the
        // roles of this kernel have to fetch as code is what slowed them all down).
        if (!masked && !__any_sync(0xffffffffu, m[0] == -INFINITY || m[1] == -INFINITY)) {
#pragma unroll 1
          for (int b = 0; b < 2; ++b) {
            uint32_t v[32], big;
            __syncwarp();
            tc::tmem_ld_16x256b_x8(ts + 64 * b, v);
            tc::tmem_ld_wait();
            float2 sum[2] = {l[0], l[1]};
            plain_weights<T>(v, sc + 64 * b, m, fac, sum, big);
            if (__any_sync(0xffffffffu, either_at_least(big, 0x7800u) || !sums_fit(sum))) {
              // The maximum has to move, by a whole power of two: what is there of this tile's weights, of O and of the
              // sums goes down by it, and the 64 weights are taken again.
              float top[2] = {-INFINITY, -INFINITY}, f[2];
              const int lo_[2] = {0, 0}, hi_[2] = {INT32_MAX, INT32_MAX};
              tc::tmem_ld_16x256b_x8(ts + 64 * b, v);
              tc::tmem_ld_wait();
              masked_top<T>(v, sc + 64 * b, fac, lo_, hi_, 0, top);
#pragma unroll
              for (int c = 0; c < 2; ++c) {
                top[c] = fmaxf(top[c], __shfl_xor_sync(0xffffffffu, top[c], 1));
                top[c] = fmaxf(top[c], __shfl_xor_sync(0xffffffffu, top[c], 2));
                const float up = floorf(fmaxf(top[c] - m[c], 0.f));
                f[c] = exp2f(-up);
                m[c] += up;
                l[c].x *= f[c], l[c].y *= f[c];
              }
              if (!(ok = before_o())) break;
              if (s > it.s0) scale_rows<DH>(tw + L::O_COL, f);
              tc::tmem_st_wait();  // the first 64 weights are read back (scale_rows has waited for them too: no tile here is an item's first)
#pragma unroll 1
              for (int part = 0; part < 2 * b; ++part) {
                uint32_t e[16];
                tc::tmem_ld_16x128b_x8(ts + 32 * part, e);
                tc::tmem_ld_wait();
#pragma unroll
                for (int k = 0; k < 16; ++k) {
                  const float2 w = __half22float2(*reinterpret_cast<const __half2*>(&e[k]));
                  e[k] = tc::pack_half2(w.x * f[k & 1], w.y * f[k & 1]);
                }
                tc::tmem_st_16x128b_x8(ts + 32 * part, e);
              }
              sum[0] = l[0], sum[1] = l[1];
              plain_weights<T>(v, sc + 64 * b, m, fac, sum, big);
            }
            l[0] = sum[0], l[1] = sum[1];
            store_weights(ts + 64 * b, v);
          }
          if (!ok) break;
        } else {  // a mask, or the item's first tile: the rows' maxima first
          float top[2] = {-INFINITY, -INFINITY};
          const int lo_[2] = {masked ? lo[0] : 0, masked ? lo[1] : 0}, hi_[2] = {masked ? hi[0] : INT32_MAX, masked ? hi[1] : INT32_MAX};
#pragma unroll 1
          for (int b = 0; b < 2; ++b) {
            uint32_t v[32];
            __syncwarp();
            tc::tmem_ld_16x256b_x8(ts + 64 * b, v);
            tc::tmem_ld_wait();
            masked_top<T>(v, sc + 64 * b, fac, lo_, hi_, key0 + 64 * b + 2 * q4, top);
          }
          const bool grow = (m[0] == -INFINITY && top[0] > -INFINITY) || top[0] > m[0] + 8.f || (m[1] == -INFINITY && top[1] > -INFINITY) ||
                            top[1] > m[1] + 8.f;
          if (__any_sync(0xffffffffu, grow)) {
            float f[2];
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              float t = top[c];
              t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 1));
              t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 2));
              t = fmaxf(m[c], t);
              f[c] = shift2(m[c], t);
              m[c] = t;
              l[c].x *= f[c], l[c].y *= f[c];
            }
            if (!(ok = before_o())) break;
            if (s > it.s0) scale_rows<DH>(tw + L::O_COL, f);
          }
          const float ref[2] = {m[0] == -INFINITY ? 0.f : m[0], m[1] == -INFINITY ? 0.f : m[1]};
#pragma unroll 1
          for (int b = 0; b < 2; ++b) {
            uint32_t v[32];
            __syncwarp();
            tc::tmem_ld_16x256b_x8(ts + 64 * b, v);
            tc::tmem_ld_wait();
            masked_weights<T>(v, sc + 64 * b, ref, fac, lo_, hi_, key0 + 64 * b + 2 * q4, l);
            store_weights(ts + 64 * b, v);
          }
        }
        tc::tmem_st_wait();
        tc::fence_before_sync();
        __syncwarp();
        if (lane == 0) {
          tc::mbar_arrive(&bars->p_full[j & 1]);  // (two tiles can be ready before P V takes the first: V may be late)
          tc::mbar_arrive(&bars->sc_empty[j % SCB]);
        }
      }
      if (!ok || !(ok = tc::mbar_wait(&bars->o_full, i & 1, abort, p.status))) break;
      tc::fence_after_sync();
      // the item's rows: output, or a part
      const bool whole = it.s0 == 0 && it.s1 == it.n && p.shared == 0;
      const int64_t slot = slot_of(p, blockIdx.x, it.part, x == x0);
      const bool fits = slot < p.list.n_slots;
      if (!whole && !fits) report(p.status, JAB_ERR_INVALID_ARG);
      float inv[2];
      int64_t out[2];
      bool live[2];
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        float t = l[c].x + l[c].y;
        t += __shfl_xor_sync(0xffffffffu, t, 1);
        t += __shfl_xor_sync(0xffffffffu, t, 2);
        const int r = r0 + g + 8 * c, rr = it.rt * R + r, q = p.by_g.quot(rr), qh = it.h * p.G + rr - q * p.G;
        const int64_t token = it.tok0 + q;
        const int64_t lse_at = token * ((int64_t)p.n_kv * p.G) + qh;
        live[c] = r < it.rows && (whole || fits);
        inv[c] = t == 0.f ? 0.f : 1.f / t;  // (of a whole item; a part stays as it is)
        out[c] = whole ? token * p.ldo + (int64_t)qh * DH : (slot * R + r) * DH;
        if (live[c]) live[c] = whole ? out_fits(p, out[c] + DH - 1, DH) && lse_fits(p, lse_at) : part_fits(p, out[c] + DH - 1, R, DH);
        if (live[c] && q4 == 0) {
          if (!whole) p.list.part_ml[slot * R + r] = make_float2(m[c], t);
          else if (p.lse != nullptr) p.lse[lse_at] = t == 0.f ? -INFINITY : (m[c] + log2f(t)) * kLn2;
        }
      }
#pragma unroll 1
      for (int b = 0; b < DH / 32; ++b) {
        uint32_t o[16];
        __syncwarp();
        tc::tmem_ld_16x256b_x4(tw + L::O_COL + 32 * b, o);
        tc::tmem_ld_wait();
        if (whole) {
          // the four lanes of a row exchange their pairs, so that each stores eight columns of its own at once
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            uint32_t w[4];
#pragma unroll
            for (int n = 0; n < 4; ++n)
              w[n] = pair_as(__uint_as_float(o[4 * n + 2 * c]) * inv[c], __uint_as_float(o[4 * n + 2 * c + 1]) * inv[c], T());
#pragma unroll
            for (int n = 0; n < 4; n += 2) {
              const uint32_t other = __shfl_xor_sync(0xffffffffu, q4 & 1 ? w[n] : w[n + 1], 1);
              w[n] = q4 & 1 ? other : w[n], w[n + 1] = q4 & 1 ? w[n + 1] : other;
            }
#pragma unroll
            for (int n = 0; n < 2; ++n) {
              const uint32_t other = __shfl_xor_sync(0xffffffffu, q4 & 2 ? w[n] : w[n + 2], 2);
              w[n] = q4 & 2 ? other : w[n], w[n + 2] = q4 & 2 ? w[n + 2] : other;
            }
            if (live[c]) *reinterpret_cast<uint4*>(static_cast<T*>(p.out) + out[c] + 32 * b + 8 * q4) = make_uint4(w[0], w[1], w[2], w[3]);
          }
        } else {
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const int c = k & 1, d = 32 * b + 8 * (k >> 1) + 2 * q4;
            if (live[c]) *reinterpret_cast<uint2*>(p.list.part_o + out[c] + d) = make_uint2(o[2 * k], o[2 * k + 1]);
          }
        }
      }
      tc::fence_before_sync();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(&bars->o_empty);
      x += it.s1 - it.s0;
    }
  } else {  // ---------------- converters
    fewer_registers<88>();
    const bool keys = warp < 16;
    const int tid = threadIdx.x - (keys ? 384 : 512);  // (of K's: row of Q, and key of a tile's scales)
    auto done = [&](uint64_t* bar) {
      tc::fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(bar);
    };
    const int total = (int)max((int64_t)0, x1 - x0);
    if (!keys) {
      for (int j = 0; j < total; ++j) {
        if (!tc::mbar_wait(&bars->rv_full[j % VST], (j / VST) & 1, abort, p.status)) break;
        if (!tc::mbar_wait(&bars->v_empty[j & 1], ((j >> 1) & 1) ^ 1, abort, p.status)) break;
        convert_tile<DH, BITS>(smem + L::RV_OFF + (j % VST) * L::RAW, smem + L::V_OFF + (j & 1) * L::TILE, tid);
        done(&bars->v_full[j & 1]);
        if (lane == 0) tc::mbar_arrive(&bars->rv_empty[j % VST]);
      }
    } else {
      const uint32_t tq = tmem + ((uint32_t)((tid >> 5) * 32) << 16) + L::Q_COL;
      int i = 0, j = 0;
      bool ok = true;
      for (int64_t x = x0; x < x1 && ok; ++i) {
        Record it;
        if (!(ok = take(i, it))) break;
        // Q of the item, once the products of the one before have read theirs
        if (!(ok = tc::mbar_wait(&bars->q_empty, (i & 1) ^ 1, abort, p.status))) break;
        tc::fence_after_sync();
        {
          const bool live = tid < it.rows;
          int lo = 0, hi = 0;  // (a row past the item's sees no key that a mask could hide: what lies there must not move the references of its warp)
          const int rr = it.rt * R + tid, q = p.by_g.quot(rr), token = it.tok0 + q;
          if (live) {
            const Entry en{it.tok0, it.nq, it.len, it.kbeg, it.all != 0};
            seen_by_row(p, en, it.all ? position_of(p, token) : it.len - it.nq + q, lo, hi);
          }
          const int64_t q_at = (int64_t)token * p.ldq + (int64_t)(it.h * p.G + rr - q * p.G) * DH;
          const uint4* row = reinterpret_cast<const uint4*>(static_cast<const T*>(p.q) + q_at);
          const bool used = live && in_bounds(q_at + DH - 1, rows_extent(p, p.ldq, DH), p.status);
          float by = 1.f, back = 1.f;
          if constexpr (std::is_same<T, bf16_t>::value) {
            uint32_t big = 0;
            if (used) {
#pragma unroll
              for (int c = 0; c < DH / 8; ++c) {
                const uint4 u = __ldg(row + c);
                big = max_abs_f16x2(max_abs_f16x2(max_abs_f16x2(max_abs_f16x2(big, u.x), u.y), u.z), u.w);
              }
            }
            row_power(max(big & 0xffffu, big >> 16) << 16, by, back);
          }
#pragma unroll
          for (int b = 0; b < DH / 64; ++b) {
            uint32_t a[32];
#pragma unroll
            for (int c = 0; c < 8; ++c) {
              uint4 u = make_uint4(0u, 0u, 0u, 0u);
              if (used) u = __ldg(row + 8 * b + c);
              uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                if constexpr (std::is_same<T, bf16_t>::value)
                  w[e] = tc::pack_half2(__uint_as_float(w[e] << 16) * by, __uint_as_float(w[e] & 0xffff0000u) * by);
                a[4 * c + e] = w[e];
              }
            }
            __syncwarp();
            tc::tmem_st32(tq + 32 * b, a);
          }
          tc::tmem_st_wait();
          // (with items of one tile, S is done with the next one's Q while the softmax writes the output of the one before)
          if (!(ok = tc::mbar_wait(&bars->rows_empty[i & 1], ((i >> 1) & 1) ^ 1, abort, p.status))) break;
          int* rows = reinterpret_cast<int*>(smem + L::ROW_OFF + (i & 1) * 3 * R * 4);
          rows[tid] = lo, rows[R + tid] = hi, rows[2 * R + tid] = __float_as_int(back);
          tc::fence_before_sync();
          __syncwarp();
          if (lane == 0) tc::mbar_arrive(&bars->q_full[i & 1]);
        }
        for (int s = it.s0; s < it.s1; ++s, ++j) {
          const uint8_t* raw = smem + L::RK_OFF + (j % KST) * L::K_STAGE;
          if (!(ok = tc::mbar_wait(&bars->rk_full[j % KST], (j / KST) & 1, abort, p.status) &&
                     tc::mbar_wait(&bars->k_empty[j & 1], ((j >> 1) & 1) ^ 1, abort, p.status) &&
                     tc::mbar_wait(&bars->sc_empty[j % SCB], ((j / SCB) & 1) ^ 1, abort, p.status)))
            break;
          const float* scales = reinterpret_cast<const float*>(raw + L::RAW);
          float* sc = reinterpret_cast<float*>(smem + L::SC_OFF + (j % SCB) * 3 * KT * 4);
          const float vs = scales[KT + tid];
          sc[tid] = scales[tid] * p.scale_log2;
          sc[KT + tid] = vs;
          sc[2 * KT + tid] = (vs < INFINITY ? fmaxf(__log2f(vs), kLeastLog2) : 0.f) - kHeadroom;
          convert_tile<DH, BITS>(raw, smem + L::K_OFF + (j & 1) * L::TILE, tid);
          done(&bars->k_full[j & 1]);
          if (lane == 0) {
            tc::mbar_arrive(&bars->sc_full[j % SCB]);
            tc::mbar_arrive(&bars->rk_empty[j % KST]);
          }
        }
        x += it.s1 - it.s0;
      }
    }
  }
  tc::fence_before_sync();
  __syncthreads();
  tc::fence_after_sync();
  if (warp == 1) {
    __syncwarp();
    tc::tmem_dealloc(tmem, 512);
  }
  if (p.behind) asm volatile("griddepcontrol.wait;" ::: "memory");
}

template <class T, int DH, int BITS>
cudaError_t launch_as(const AttnParams& p, int64_t est_tiles, int sms, cudaStream_t st) {
  using L = Layout<DH, BITS>;
  auto kern = kv_tile_kernel<T, DH, BITS>;
  constexpr int most = L::USED + 1024 + 2 * 2050 * 4;
  static_assert(most <= 226 * 1024 + 512, "shared memory budget");
  const int smem = L::USED + 1024 + 2 * (p.n_seqs + 2) * 4;
  static SetUp ready;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  e = ready.once(dev, [&] { return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, most); });
  if (e != cudaSuccess) return e;
  const int64_t grid = std::max<int64_t>(1, std::min<int64_t>(sms, est_tiles));
  return launch_after(kern, (unsigned)grid, THREADS, (size_t)smem, st, p);
}

template <class T>
cudaError_t launch_type(const AttnParams& p, int dh, int bits, int64_t est, int sms, cudaStream_t st) {
  if (dh == 128) return bits == 8 ? launch_as<T, 128, 8>(p, est, sms, st) : launch_as<T, 128, 4>(p, est, sms, st);
  return bits == 8 ? launch_as<T, 64, 8>(p, est, sms, st) : launch_as<T, 64, 4>(p, est, sms, st);
}

}  // namespace

cudaError_t launch_tiles(const AttnParams& p, jab_dtype type, int dh, int bits, int64_t est_tiles, int sms, cudaStream_t st) {
  return type == JAB_FP16 ? launch_type<half_t>(p, dh, bits, est_tiles, sms, st) : launch_type<bf16_t>(p, dh, bits, est_tiles, sms, st);
}

}  // namespace kv
}  // namespace jab
