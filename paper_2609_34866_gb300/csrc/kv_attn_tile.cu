// Attention over the quantised paged cache for many rows that see the same keys (chunks of a prompt, a prefix that
// all sequences share): 128 rows x 128 keys at a time on the tensor cores, by the formulas of kv_attn.cu.
//
// The codes of a key tile come as the bytes that they are, by bulk copies of 16 keys (a page holds whole groups of
// 16), and become fp16 in shared memory once per tile; the scales stay outside of the products as they do there.
// Both products are M128 N128 with their A operand in tensor memory:
//   S = Q K^T   A = Q (fp16, written to tensor memory row by row), B = K as converted (K-major)
//   O += P V    A = P (fp16 weights, written by the softmax), B = V as converted (MN-major: the same layout)
// In key tiles that a mask cuts, P is its fp16 value and what that leaves over, in two products: rows that see few
// keys (the first of a sequence, narrow windows) have them in such tiles, and one rounding of a weight would
// show. In the others a weight is rounded once (2^-11 of it at most, over 128 keys and more).
//   warp 0        bulk copies: 8 groups of K, V and their scales a tile, one copy per lane; ring of RST tiles
//   warp 1        tensor memory owner; issues S, a tile ahead of P V;   warp 2  issues P V
//   warps 4..11   softmax: 16 rows a warp, four threads a row (16x256b shape); at an item's end the output
//   warps 12..15  converters: Q of the next item, then per tile K (one ahead), V, and the keys' scales
#include <algorithm>
#include <type_traits>

#include "kv_attn.cuh"
#include "tc.cuh"

namespace jab {
namespace kv {
namespace {

constexpr int R = kTileRows, KT = kTileKeys, THREADS = 512, RST = 2, SCB = 3;

template <int DH, int BITS>
struct Layout {
  static constexpr int CHUNK = 128 * 128;              // 128 keys x 64 dimensions of fp16, 128-byte swizzle
  static constexpr int TILE = KT * DH * 2;             // K or V in fp16
  static constexpr int RAW = KT * DH * BITS / 8;       // K or V as codes
  static constexpr int STAGE = 2 * RAW + 2 * KT * 4;   // K, V, scales of K, of V
  static constexpr int K_OFF = 0, V_OFF = 2 * TILE, RAW_OFF = 3 * TILE;
  static constexpr int SC_OFF = RAW_OFF + RST * STAGE;            // per tile: K scale * log2 e * c, V scale, its log2
  static constexpr int ROW_OFF = SC_OFF + SCB * 3 * KT * 4;       // per item: lo, hi, power of two of Q
  static constexpr int BAR_OFF = ROW_OFF + 2 * 3 * R * 4;
  static constexpr int USED = BAR_OFF + 512;
  static constexpr uint32_t S_COL = 0, O_COL = 128, Q_COL = 256, P_COL = 320, LO_COL = 384;
};

struct Bars {
  uint64_t raw_full[RST], raw_empty[RST], k_full[2], k_empty[2], sc_full[SCB], v_full;
  uint64_t q_full[2], q_empty, s_full, s_empty, p_full, pv_done, o_full, o_empty, drain[2];
  uint32_t tmem_base;
  int abort;
};
static_assert(sizeof(Bars) <= 512, "barrier block");

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

// 8 codes (8 or 4 bytes at src) as fp16, in their order.
template <int BITS>
__device__ __forceinline__ uint4 eight_codes(const uint8_t* src) {
  uint4 r;
  if constexpr (BITS == 8) {
    const uint2 w = *reinterpret_cast<const uint2*>(src);
    constexpr uint32_t k = 0x64806480u;  // 1152
    r.x = biased_h2(__byte_perm(w.x, 0x64646464u, 0x4140), k);
    r.y = biased_h2(__byte_perm(w.x, 0x64646464u, 0x4342), k);
    r.z = biased_h2(__byte_perm(w.y, 0x64646464u, 0x4140), k);
    r.w = biased_h2(__byte_perm(w.y, 0x64646464u, 0x4342), k);
  } else {
    const uint32_t w = *reinterpret_cast<const uint32_t*>(src);
    constexpr uint32_t k = 0x64086408u;  // 1032
    const uint32_t even = w & 0x0f0f0f0fu, odd = (w >> 4) & 0x0f0f0f0fu;
    const uint32_t a = __byte_perm(even, odd, 0x5140), b = __byte_perm(even, odd, 0x7362);
    r.x = biased_h2(__byte_perm(a, 0x64646464u, 0x4140), k);
    r.y = biased_h2(__byte_perm(a, 0x64646464u, 0x4342), k);
    r.z = biased_h2(__byte_perm(b, 0x64646464u, 0x4140), k);
    r.w = biased_h2(__byte_perm(b, 0x64646464u, 0x4342), k);
  }
  return r;
}

// A tile of codes to fp16 in the swizzled layout, by 128 threads: consecutive threads take consecutive eights of a
// row, so that reads and 16-byte writes are free of bank conflicts.
template <int DH, int BITS>
__device__ __forceinline__ void convert_tile(const uint8_t* raw, uint8_t* dst, int tid) {
  constexpr int PER_ROW = DH / 8;
#pragma unroll 4
  for (int i = tid; i < KT * PER_ROW; i += 128) {
    const int key = i / PER_ROW, c = i % PER_ROW;
    *reinterpret_cast<uint4*>(dst + (c >> 3) * (128 * 128) + key * 128 + (((c & 7) ^ (key & 7)) << 4)) =
        eight_codes<BITS>(raw + i * BITS);
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
    for (int s = 0; s < RST; ++s) {
      tc::mbar_init(&bars->raw_full[s], 1);
      tc::mbar_init(&bars->raw_empty[s], 4);
    }
    for (int s = 0; s < 2; ++s) {
      tc::mbar_init(&bars->k_full[s], 4);
      tc::mbar_init(&bars->k_empty[s], 1);
      tc::mbar_init(&bars->drain[s], 1);
      tc::mbar_init(&bars->q_full[s], 4);
    }
    for (int s = 0; s < SCB; ++s) tc::mbar_init(&bars->sc_full[s], 4);
    tc::mbar_init(&bars->v_full, 4);
    tc::mbar_init(&bars->q_empty, 1);
    tc::mbar_init(&bars->s_full, 1);
    tc::mbar_init(&bars->s_empty, 8);
    tc::mbar_init(&bars->p_full, 8);
    tc::mbar_init(&bars->pv_done, 1);
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
  stream_order();
  make_plan<R, KT, THREADS / 32, 1>(p, cum_t, cum_i, head);
  const int64_t all = (int64_t)head[kTotal] * p.n_kv;
  const int64_t x0 = (int64_t)blockIdx.x * head[kPer], x1 = min(all, x0 + head[kPer]);
  // Every role walks the block's items; j counts key tiles and i items over all of them.
  if (warp < 4) {
    fewer_registers<64>();
    if (warp == 0) {  // ---------------- bulk copies
      int j = 0;
      bool ok = true;
      const int kind = lane >> 3, grp = lane & 7;  // K, V, scales of K, of V; group of 16 keys
      const uint8_t* src = kind == 0   ? p.k_codes
                           : kind == 1 ? p.v_codes
                           : kind == 2 ? reinterpret_cast<const uint8_t*>(p.k_scales)
                                       : reinterpret_cast<const uint8_t*>(p.v_scales);
      constexpr int ROW = DH * BITS / 8;
      const int row_bytes = kind < 2 ? ROW : 4;
      const int off = kind < 2 ? kind * L::RAW : 2 * L::RAW + (kind - 2) * KT * 4;
      for (int64_t x = x0; x < x1 && ok;) {
        const Item it = item_at<R, KT>(p, cum_t, head, x, x1);
        const int32_t* table = p.pages + (it.en.all ? 0 : (int64_t)(it.e - (p.list.all ? 1 : 0)) * p.max_pages);
        for (int s = it.s0; s < it.s1; ++s, ++j) {
          const int st = j % RST;
          const int key = (it.t0 + s) * KT + grp * 16;
          const bool have = key < it.en.len;  // (what lies past the keys is hidden, whatever is in its place)
          int64_t row = 0;
          if (have) {
            const int pg = p.by_page.quot(key);
            int id = __ldg(table + pg);
            if (id < 0 || id >= p.n_pages) {
              report(p.status, JAB_ERR_INVALID_ARG);
              id = 0;
            }
            row = ((int64_t)id * p.n_kv + it.h) * p.page + (key - pg * p.page);
          }
          ok = tc::mbar_wait(&bars->raw_empty[st], ((j / RST) & 1) ^ 1, abort, p.status);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          const unsigned n = __popc(__ballot_sync(0xffffffffu, have) & 0xffu);
          if (lane == 0) tc::mbar_expect_tx(&bars->raw_full[st], n * 16 * (2 * ROW + 8));
          __syncwarp();
          if (have)
            tc::bulk_load(smem + L::RAW_OFF + st * L::STAGE + off + grp * 16 * row_bytes, src + row * row_bytes, 16 * row_bytes,
                          &bars->raw_full[st]);
        }
        x += it.s1 - it.s0;
      }
      if (*abort)
        for (int k = max(0, j - RST); k < j; ++k) drain_wait(&bars->raw_full[k % RST], (k / RST) & 1);
    } else if (warp == 1 && tc::elect_one()) {  // ---------------- S
      constexpr uint32_t IDESC = tc::idesc_f16(false, R, KT);
      int j = 0, i = 0;
      bool ok = true;
      for (int64_t x = x0; x < x1 && ok; ++i) {
        const Item it = item_at<R, KT>(p, cum_t, head, x, x1);
        ok = tc::mbar_wait(&bars->q_full[i & 1], (i >> 1) & 1, abort, p.status);
        for (int s = it.s0; s < it.s1 && ok; ++s, ++j) {
          ok = tc::mbar_wait(&bars->k_full[j & 1], (j >> 1) & 1, abort, p.status) &&
               tc::mbar_wait(&bars->s_empty, (j & 1) ^ 1, abort, p.status);
          if (!ok) break;
          tc::fence_after_sync();
          const uint64_t kd = tc::sdesc_kmajor_sw128(tc::smem_u32(smem + L::K_OFF + (j & 1) * L::TILE));
#pragma unroll
          for (int k = 0; k < DH / 16; ++k)
            tc::umma_f16_ts(tmem + L::S_COL, tmem + L::Q_COL + k * 8, tc::sdesc_advance(kd, (k >> 2) * L::CHUNK + (k & 3) * 32), IDESC,
                            k > 0 ? 1u : 0u);
          tc::umma_commit(&bars->s_full);
          tc::umma_commit(&bars->k_empty[j & 1]);
        }
        if (ok) tc::umma_commit(&bars->q_empty);
        x += it.s1 - it.s0;
      }
      tc::umma_commit(&bars->drain[0]);
      drain_wait(&bars->drain[0], 0);
    } else if (warp == 2 && tc::elect_one()) {  // ---------------- P V
      constexpr uint32_t IDESC = tc::idesc_f16(false, R, DH) | (1u << 16);  // B MN-major
      int j = 0, i = 0;
      bool ok = true;
      const uint64_t vd = tc::sdesc_mnmajor_sw128(tc::smem_u32(smem + L::V_OFF), L::CHUNK, 1024);
      for (int64_t x = x0; x < x1 && ok; ++i) {
        const Item it = item_at<R, KT>(p, cum_t, head, x, x1);
        int all_lo, all_hi;
        seen_by_all(p, it.en, it.rt * R, it.rt * R + it.rows, head, all_lo, all_hi);
        ok = tc::mbar_wait(&bars->o_empty, (i & 1) ^ 1, abort, p.status);
        for (int s = it.s0; s < it.s1 && ok; ++s, ++j) {
          ok = tc::mbar_wait(&bars->v_full, j & 1, abort, p.status) && tc::mbar_wait(&bars->p_full, j & 1, abort, p.status);
          if (!ok) break;
          tc::fence_after_sync();
          const int key0 = (it.t0 + s) * KT;
          const bool masked = key0 < all_lo || key0 + KT > all_hi;
#pragma unroll
          for (int k = 0; k < KT / 16; ++k)
            tc::umma_f16_ts(tmem + L::O_COL, tmem + L::P_COL + k * 8, tc::sdesc_advance(vd, k * 16 * 128), IDESC,
                            s > it.s0 || k > 0 ? 1u : 0u);
          if (masked) {
#pragma unroll
            for (int k = 0; k < KT / 16; ++k)
              tc::umma_f16_ts(tmem + L::O_COL, tmem + L::LO_COL + k * 8, tc::sdesc_advance(vd, k * 16 * 128), IDESC, 1u);
          }
          tc::umma_commit(&bars->pv_done);
        }
        if (ok) tc::umma_commit(&bars->o_full);
        x += it.s1 - it.s0;
      }
      tc::umma_commit(&bars->drain[1]);
      drain_wait(&bars->drain[1], 0);
    }
  } else if (warp < 12) {  // ---------------- softmax
    more_registers<168>();
    const int quarter = warp & 3, g = lane >> 2, q4 = lane & 3;
    const int r0 = 32 * quarter + 16 * ((warp - 4) >> 2);  // the warp's first row
    const uint32_t tw = tmem + ((uint32_t)r0 << 16);
    int j = 0, i = 0;
    bool ok = true;
    for (int64_t x = x0; x < x1 && ok; ++i) {
      const Item it = item_at<R, KT>(p, cum_t, head, x, x1);
      int all_lo, all_hi;
      seen_by_all(p, it.en, it.rt * R, it.rt * R + it.rows, head, all_lo, all_hi);
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
      for (int s = it.s0; s < it.s1; ++s, ++j) {
        const float* sc = reinterpret_cast<const float*>(smem + L::SC_OFF + (j % SCB) * 3 * KT * 4) + 2 * q4;
        if (!(ok = tc::mbar_wait(&bars->sc_full[j % SCB], (j / SCB) & 1, abort, p.status) &&
                   tc::mbar_wait(&bars->s_full, j & 1, abort, p.status)))
          break;
        tc::fence_after_sync();
        uint32_t v[2][32];
        __syncwarp();
        tc::tmem_ld_16x256b_x8(tw + L::S_COL, v[0]);
        tc::tmem_ld_16x256b_x8(tw + L::S_COL + 64, v[1]);
        tc::tmem_ld_wait();
        tc::fence_before_sync();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&bars->s_empty);
        const int key0 = (it.t0 + s) * KT;
        const bool masked = key0 < all_lo || key0 + KT > all_hi;
        // y = score - m (m: the maximum so far, of score + log2 of the key's V scale)
        const float ref[2] = {m[0] == -INFINITY ? 0.f : m[0], m[1] == -INFINITY ? 0.f : m[1]};
        float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int n = 0; n < 16; ++n) {
          const float2 ks = *reinterpret_cast<const float2*>(sc + 8 * n), lv = *reinterpret_cast<const float2*>(sc + 2 * KT + 8 * n);
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            uint32_t* e = &v[n >> 3][4 * (n & 7) + 2 * c];
            float2 a = make_float2(__uint_as_float(e[0]), __uint_as_float(e[1]));
            if constexpr (std::is_same<T, bf16_t>::value) a = tc::mul2(a, make_float2(fac[c], fac[c]));
            float2 y = tc::fma2(a, ks, make_float2(-ref[c], -ref[c]));
            if (masked) {
              const int k = key0 + 8 * n + 2 * q4;
              if (k < lo[c] || k >= hi[c]) y.x = -INFINITY;
              if (k + 1 < lo[c] || k + 1 >= hi[c]) y.y = -INFINITY;
              // (a hidden key's scales may be anything)
              if (y.x != -INFINITY) top[c] = fmaxf(top[c], y.x + lv.x);
              if (y.y != -INFINITY) top[c] = fmaxf(top[c], y.y + lv.y);
            } else {
              const float2 u = tc::add2(y, lv);
              top[c] = tc::fmax3(top[c], u.x, u.y);
            }
            e[0] = __float_as_uint(y.x), e[1] = __float_as_uint(y.y);
          }
        }
        // P V of the tile before is done: O may be rescaled and P written
        if (j > 0 && !(ok = tc::mbar_wait(&bars->pv_done, (j - 1) & 1, abort, p.status))) break;
        tc::fence_after_sync();
        const bool grow = (m[0] == -INFINITY && top[0] > -INFINITY) || top[0] > 8.f || (m[1] == -INFINITY && top[1] > -INFINITY) || top[1] > 8.f;
        if (__any_sync(0xffffffffu, grow)) {
          float f[2], d[2];
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            float t = top[c];
            t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 1));
            t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 2));
            const float mn = fmaxf(m[c], ref[c] + t);
            f[c] = shift2(m[c], mn);
            d[c] = mn == -INFINITY ? 0.f : ref[c] - mn;
            m[c] = mn;
            l[c].x *= f[c], l[c].y *= f[c];
          }
#pragma unroll
          for (int n = 0; n < 32; ++n) {
            v[n >> 4][2 * (n & 15)] = __float_as_uint(__uint_as_float(v[n >> 4][2 * (n & 15)]) + d[n & 1]);
            v[n >> 4][2 * (n & 15) + 1] = __float_as_uint(__uint_as_float(v[n >> 4][2 * (n & 15) + 1]) + d[n & 1]);
          }
          if (s > it.s0) {
#pragma unroll
            for (int b = 0; b < DH / 32; ++b) {
              uint32_t o[16];
              tc::tmem_ld_16x256b_x4(tw + L::O_COL + 32 * b, o);
              tc::tmem_ld_wait();
#pragma unroll
              for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * f[(k >> 1) & 1]);
              tc::tmem_st_16x256b_x4(tw + L::O_COL + 32 * b, o);
            }
            tc::tmem_st_wait();
          }
        }
        // weights
        uint32_t hi2[32], lo2[32];
#pragma unroll
        for (int n = 0; n < 16; ++n) {
          const float2 vs = *reinterpret_cast<const float2*>(sc + KT + 8 * n);
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            const uint32_t* e = &v[n >> 3][4 * (n & 7) + 2 * c];
            const float2 ex = make_float2(tc::fast_exp2(__uint_as_float(e[0])), tc::fast_exp2(__uint_as_float(e[1])));
            l[c] = tc::add2(l[c], ex);
            float2 w = tc::mul2(ex, vs);
            if (masked) {
              if (__uint_as_float(e[0]) == -INFINITY) w.x = 0.f;
              if (__uint_as_float(e[1]) == -INFINITY) w.y = 0.f;
            }
            const uint32_t h = tc::pack_half2(w.x, w.y);
            hi2[2 * n + c] = h;
            if (masked) {
              const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
              lo2[2 * n + c] = tc::pack_half2(w.x - f.x, w.y - f.y);
            }
          }
        }
        __syncwarp();
        tc::tmem_st_16x128b_x16(tw + L::P_COL, hi2);
        if (masked) tc::tmem_st_16x128b_x16(tw + L::LO_COL, lo2);
        tc::tmem_st_wait();
        tc::fence_before_sync();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&bars->p_full);
      }
      if (!ok || !(ok = tc::mbar_wait(&bars->o_full, i & 1, abort, p.status))) break;
      tc::fence_after_sync();
      // the item's rows: output, or a part
      const bool whole = it.s0 == 0 && it.s1 == it.n && p.shared == 0;
      const int64_t slot = slot_of(p, blockIdx.x, it.h * head[kItems] + cum_i[it.e] + it.rt, x == x0);
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
        const int64_t token = it.en.tok0 + q;
        live[c] = r < it.rows && (whole || fits);
        inv[c] = whole ? (t == 0.f ? 0.f : 1.f / t) : 1.f;
        out[c] = whole ? token * p.ldo + (int64_t)qh * DH : (slot * R + r) * DH;
        if (live[c] && q4 == 0) {
          if (!whole) p.list.part_ml[slot * R + r] = make_float2(m[c], t);
          else if (p.lse != nullptr) p.lse[token * ((int64_t)p.n_kv * p.G) + qh] = t == 0.f ? -INFINITY : (m[c] + log2f(t)) * kLn2;
        }
      }
#pragma unroll
      for (int b = 0; b < DH / 32; ++b) {
        uint32_t o[16];
        __syncwarp();
        tc::tmem_ld_16x256b_x4(tw + L::O_COL + 32 * b, o);
        tc::tmem_ld_wait();
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const int c = k & 1, d = 32 * b + 8 * (k >> 1) + 2 * q4;
          const float a0 = __uint_as_float(o[2 * k]) * inv[c], a1 = __uint_as_float(o[2 * k + 1]) * inv[c];
          if (!live[c]) continue;
          if (whole) {
            T two[2];
            store_out(two, a0), store_out(two + 1, a1);
            *reinterpret_cast<uint32_t*>(static_cast<T*>(p.out) + out[c] + d) = *reinterpret_cast<const uint32_t*>(two);
          } else {
            *reinterpret_cast<float2*>(p.list.part_o + out[c] + d) = make_float2(a0, a1);
          }
        }
      }
      tc::fence_before_sync();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(&bars->o_empty);
      x += it.s1 - it.s0;
    }
  } else {  // ---------------- converters
    fewer_registers<96>();
    const int tid = threadIdx.x - 384;  // row of Q, and key of a tile's scales
    const uint32_t tq = tmem + ((uint32_t)((tid >> 5) * 32) << 16) + L::Q_COL;
    auto raw_of = [&](int k) { return smem + L::RAW_OFF + (k % RST) * L::STAGE; };
    auto done = [&](uint64_t* bar) {
      tc::fence_proxy_async_smem();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(bar);
    };
    // K and the scales of tile k
    auto keys_of = [&](int k) -> bool {
      if (!tc::mbar_wait(&bars->raw_full[k % RST], (k / RST) & 1, abort, p.status) ||
          !tc::mbar_wait(&bars->k_empty[k & 1], ((k >> 1) & 1) ^ 1, abort, p.status))
        return false;
      const uint8_t* raw = raw_of(k);
      const float* ksv = reinterpret_cast<const float*>(raw + 2 * L::RAW);
      float* sc = reinterpret_cast<float*>(smem + L::SC_OFF + (k % SCB) * 3 * KT * 4);
      const float vs = ksv[KT + tid];
      sc[tid] = ksv[tid] * p.scale_log2;
      sc[KT + tid] = vs;
      sc[2 * KT + tid] = vs > 0.f ? __log2f(vs) : vs == 0.f ? -100.f : vs;  // (a row of zeros counts as one of 2^-100)
      done(&bars->sc_full[k % SCB]);
      convert_tile<DH, BITS>(raw, smem + L::K_OFF + (k & 1) * L::TILE, tid);
      done(&bars->k_full[k & 1]);
      return true;
    };
    int j = 0, i = 0;
    bool ok = true;
    const int total = (int)max((int64_t)0, x1 - x0);
    for (int64_t x = x0; x < x1 && ok; ++i) {
      const Item it = item_at<R, KT>(p, cum_t, head, x, x1);
      // Q of this item, once the products of the one before have read theirs; its rows' bounds
      if (!(ok = tc::mbar_wait(&bars->q_empty, (i & 1) ^ 1, abort, p.status))) break;
      tc::fence_after_sync();
      {
        const bool live = tid < it.rows;
        int lo = 0, hi = INT32_MAX;
        const int rr = it.rt * R + tid, q = p.by_g.quot(rr), token = it.en.tok0 + q;
        if (live) seen_by_row(p, it.en, it.en.all ? position_of(p, token) : it.en.len - it.en.nq + q, lo, hi);
        const uint4* row = reinterpret_cast<const uint4*>(static_cast<const T*>(p.q) + (int64_t)token * p.ldq + (int64_t)(it.h * p.G + rr - q * p.G) * DH);
        float by = 1.f, back = 1.f;
        if constexpr (std::is_same<T, bf16_t>::value) {
          uint32_t big = 0;
          if (live) {
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
            if (live) u = __ldg(row + 8 * b + c);
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
        int* rows = reinterpret_cast<int*>(smem + L::ROW_OFF + (i & 1) * 3 * R * 4);
        rows[tid] = lo, rows[R + tid] = hi, rows[2 * R + tid] = __float_as_int(back);
        tc::fence_before_sync();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&bars->q_full[i & 1]);
      }
      if (j == 0 && !(ok = keys_of(0))) break;
      for (int s = it.s0; s < it.s1; ++s, ++j) {
        if (j + 1 < total && !(ok = keys_of(j + 1))) break;
        if (j > 0 && !(ok = tc::mbar_wait(&bars->pv_done, (j - 1) & 1, abort, p.status))) break;
        convert_tile<DH, BITS>(raw_of(j) + L::RAW, smem + L::V_OFF, tid);
        done(&bars->v_full);
        if (lane == 0) tc::mbar_arrive(&bars->raw_empty[j % RST]);
      }
      x += it.s1 - it.s0;
    }
  }
  tc::fence_before_sync();
  __syncthreads();
  tc::fence_after_sync();
  if (warp == 1) {
    __syncwarp();
    tc::tmem_dealloc(tmem, 512);
  }
}

template <class T, int DH, int BITS>
cudaError_t launch_as(const AttnParams& p, int64_t est_tiles, int sms, cudaStream_t st) {
  using L = Layout<DH, BITS>;
  auto kern = kv_tile_kernel<T, DH, BITS>;
  constexpr int most = L::USED + 1024 + 2 * 4098 * 4;
  static_assert(most <= 226 * 1024, "shared memory budget");
  const int smem = L::USED + 1024 + 2 * (p.n_seqs + 2) * 4;
  static bool attr_set = false;
  if (!attr_set) {
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, most);
    if (e != cudaSuccess) return e;
    attr_set = true;
  }
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
