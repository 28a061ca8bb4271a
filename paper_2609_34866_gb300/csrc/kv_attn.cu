// Attention of new tokens over the quantised paged cache (single tokens, short runs of them, chunks).
//
//   s_ij = c k_j (q_i . K_j)          K_j, V_j whole numbers (codes), k_j, v_j their scales,
//   w_ij = 2^(s_ij - m_i) v_j         c = softmax scale * log2 e
//   o_i  = sum_j w_ij V_j / sum_j 2^(s_ij - m_i)
//
// The codes are exact in fp16 and the scales stay outside of the products: the one on K multiplies the
// score, the one on V the weight, so a byte of the cache costs one or two integer instructions and one
// subtraction on its way to the matrix instructions. m_i is a running maximum of s_ij + log2 v_j - 6, not of
// s_ij: the weights that are rounded to fp16 are then at most 2^15 whatever the scales of V are.
//
// Rows of a tile are (token, query head) pairs that share a KV head, R = 8 NT of them. Keys go 16 at a time, two such
// groups together:
// S^T = K Q^T and O^T = V^T P^T by m16n8k16 products with the cache's side as the 16-row operand, because a
// decoding step has few rows (4 for a GQA ratio of 4: half of n8 idle, where they would leave three quarters
// of m16). No operand is rearranged on its way: the dimensions that a sum runs over may be permuted, so a lane takes
// head_dim / 4 consecutive codes of its K row, and head_dim / 8 of each of its four V rows.
//
// Work is cut into equal numbers of key tiles over warps that are resident at once, whatever the lengths (kv_attn.cuh);
// a warp takes its share by itself, with no barrier, its copies running ahead of it across the share's items. Keys
// shared by all sequences are one more entry of the list, whose rows are those of all sequences. A second kernel
// joins the parts of items that went to several warps.
//
// Bound: the cache's bytes; 64 sequences of up to 8192 keys of 8 heads of 128 (328 MB) are read at 5.2 TB/s in 63 us, joined
// in 10. In 4 bits the conversion of codes takes as long as their bytes would (4 sequences of up to 65536 keys, 227 MB:
// 3.5 TB/s with 51 % of the issue slots in use).
#include <algorithm>
#include <type_traits>

#include "kv_attn.cuh"
#include "per_device.h"
#include "tc.cuh"

namespace jab {
namespace kv {
namespace {

constexpr int W = 4;  // warps of a block

// ------------------------------------------------------------------ codes to fp16
// A byte b under the exponent of 1024 is 1024 + b; less 1152 it is b - 128.
__device__ __forceinline__ uint32_t sub_h2(uint32_t a, uint32_t b) {
  const __half2 r = __hsub2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
  return *reinterpret_cast<const uint32_t*>(&r);
}
__device__ __forceinline__ uint32_t fma_h2(uint32_t a, uint32_t b, uint32_t c) {
  const __half2 r = __hfma2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b), *reinterpret_cast<const __half2*>(&c));
  return *reinterpret_cast<const uint32_t*>(&r);
}
constexpr uint32_t k1152 = 0x64806480u, k1032 = 0x64086408u, kSixteenth = 0x2c002c00u, kMinus72 = 0xd480d480u;

// bytes (0, 1) and (2, 3) of w as fp16 pairs
__device__ __forceinline__ void bytes_h2(uint32_t w, uint32_t& lo, uint32_t& hi) {
  lo = sub_h2(__byte_perm(w, 0x64646464u, 0x4140), k1152);
  hi = sub_h2(__byte_perm(w, 0x64646464u, 0x4342), k1152);
}
// nibbles (j, j + 4) of w as fp16 pairs, j = 0 .. 3: those at bits 4 of a byte stand for 16 times as much
__device__ __forceinline__ void nibbles_h2(uint32_t w, uint32_t (&r)[4]) {
  const uint32_t u = w >> 8;
  r[0] = sub_h2((w & 0x000f000fu) | 0x64006400u, k1032);
  r[1] = fma_h2((w & 0x00f000f0u) | 0x64006400u, kSixteenth, kMinus72);
  r[2] = sub_h2((u & 0x000f000fu) | 0x64006400u, k1032);
  r[3] = fma_h2((u & 0x00f000f0u) | 0x64006400u, kSixteenth, kMinus72);
}

__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t a) {
  uint32_t d;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
  return d;
}

// A key tile, NS groups of 16 keys, in shared memory, where DEPTH of them wait for their warp: rows as they are in the
// cache (V's of a group in the order (0, 2, 4, 6), (1, 3, 5, 7), (8, ...), (9, ...), as the lanes take them), their
// 16-byte pieces exchanged so that neither the copies nor the reads meet in a bank; then a pair of scales per key.
// Copies go along the rows, whole lines at a time: by the lanes that use the bytes, 4 rows of V an eighth of the warp,
// they took 59 us where these took 40 (64 sequences of up to 8192 keys, arithmetic left out for the comparison).
constexpr int DEPTH = 2;
template <int DH, int BITS, int NS>
struct Tile {
  static constexpr int ROW = DH * BITS / 8, KB = ROW / 4, VB = ROW / 8;
  static constexpr int KU = KB < 16 ? KB : 16;  // bytes of a read of K
  static constexpr int GROUP = 16 * ROW, V_OFF = NS * GROUP, S_OFF = 2 * NS * GROUP, BYTES = S_OFF + NS * 16 * 8;
  // Place of byte `b` of row r (of V: of the r-th in the order above).
  static __device__ __forceinline__ int k_at(int r, int b) { return r * ROW + (ROW == 128 ? b ^ ((r & 1) << 6) : b); }
  static __device__ __forceinline__ int v_at(int r, int b) {
    return r * ROW + (ROW == 128 ? b ^ ((r & 3) << 5) : ROW == 64 ? b ^ ((r & 2) << 4) : b);
  }
};

template <int N>
__device__ __forceinline__ void copy_async(uint32_t dst, const void* src) {
  if constexpr (N == 16)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
  else
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(src), "n"(N) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// What a lane copies of every tile: the constant parts of its addresses.
template <int DH, int BITS, int NS>
struct CopyLane {
  using TT = Tile<DH, BITS, NS>;
  static constexpr int PER_ROW = TT::ROW / 16, STEP = 32 / PER_ROW;  // pieces of a row, rows of a copy
  const uint8_t *k, *v;
  const float* scales;
  uint32_t k_to, v_to[16 / STEP], s_to;
  __device__ __forceinline__ CopyLane(const AttnParams& p, int lane, uint32_t queue) {
    const int r0 = lane / PER_ROW, byte = lane % PER_ROW * 16;
    k = p.k_codes + lane * 16;
    v = p.v_codes + lane * 16;
    k_to = queue + TT::k_at(r0, byte);  // (rows STEP apart have the same parity)
#pragma unroll
    for (int i = 0; i < 16 / STEP; ++i) {
      const int row = r0 + i * STEP;
      v_to[i] = queue + TT::V_OFF + TT::v_at(((row & 1) + 2 * (row >> 3)) * 4 + ((row >> 1) & 3), byte);
    }
    // scales: key `lane` of the tile, K's and V's; with one group V's are the upper half warp's
    const bool upper = NS == 1 && lane >= 16;
    scales = (upper ? p.v_scales : p.k_scales) + (lane & 15);
    s_to = queue + TT::S_OFF + (lane & (NS * 16 - 1)) * 8 + (upper ? 4 : 0);
  }
  // rows: places of the tile's groups in the cache, in groups of 16 rows; at: the tile's place in the queue.
  __device__ __forceinline__ void copy(const AttnParams& p, const int (&rows)[NS], int lane, uint32_t at) const {
#pragma unroll
    for (int n = 0; n < NS; ++n) {
      const int64_t base = (int64_t)rows[n] * TT::GROUP;
#pragma unroll
      for (int i = 0; i < 16 / STEP; ++i) {
        copy_async<16>(at + k_to + (n * TT::GROUP + i * 512), k + base + i * 512);
        copy_async<16>(at + v_to[i] + n * TT::GROUP, v + base + i * 512);
      }
    }
    const int64_t row = (int64_t)(NS == 2 && lane >= 16 ? rows[NS - 1] : rows[0]) << 4;
    copy_async<4>(at + s_to, scales + row);
    if (NS == 2) copy_async<4>(at + s_to + 4, p.v_scales + (lane & 15) + row);
  }
};

// U bytes at p as 32-bit words.
template <int U>
__device__ __forceinline__ void take(const uint8_t* p, uint32_t* w) {
  if constexpr (U == 16) {
    const uint4 v = *reinterpret_cast<const uint4*>(p);
    w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
  } else if constexpr (U == 8) {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    w[0] = v.x, w[1] = v.y;
  } else {
    w[0] = *reinterpret_cast<const uint32_t*>(p);
  }
}

// Q's dimensions that go with a lane's codes of K, as the B operand of K's steps; returns the power of two that the row
// was divided by (bf16: it is brought into fp16's range; exact down to 2^-31 of its largest). A lane has DH / 4 of them, in
// runs of what it reads at once.
template <class T, int DH, int BITS>
__device__ __forceinline__ float load_q(const T* row, int q, bool live, uint32_t (&b)[DH / 8]) {
  float f[DH / 4];
  constexpr int RUN = Tile<DH, BITS, 1>::KU * 8 / BITS;  // dimensions of a copy
#pragma unroll
  for (int i = 0; i < DH / 4; i += 8) {
    uint4 u = make_uint4(0u, 0u, 0u, 0u);
    if (live) u = __ldg(reinterpret_cast<const uint4*>(row + (i / RUN) * 4 * RUN + q * RUN + i % RUN));
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (std::is_same<T, half_t>::value) {
        const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&w[j]));
        f[i + 2 * j] = x.x, f[i + 2 * j + 1] = x.y;
      } else {
        f[i + 2 * j] = __uint_as_float(w[j] << 16), f[i + 2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
      }
    }
  }
  float back = 1.f;
  if constexpr (!std::is_same<T, half_t>::value) {
    uint32_t big = 0;
#pragma unroll
    for (int i = 0; i < DH / 4; ++i) big = max(big, __float_as_uint(f[i]) & 0x7fffffffu);
    big = max(big, __shfl_xor_sync(0xffffffffu, big, 1));
    big = max(big, __shfl_xor_sync(0xffffffffu, big, 2));
    float by;
    row_power(big, by, back);
#pragma unroll
    for (int i = 0; i < DH / 4; ++i) f[i] *= by;
  }
#pragma unroll
  for (int i = 0; i < DH / 8; ++i) {
    // 8 bits: elements in their order; 4 bits: (j, j + 4) of each eight
    const int a = BITS == 8 ? 2 * i : 8 * (i / 4) + (i & 3), c = BITS == 8 ? a + 1 : a + 4;
    b[i] = tc::pack_half2(f[a], f[c]);
  }
  return back;
}

// Weights of a tile's scores s (of every group keys g, g + 8; rows 2q, 2q + 1 of each eight): their sums in l, and the
// weights as B operands of V's products. m, l and o follow when the maximum has grown by more than 2^8. sc: the
// keys' scales. MASKED: rows see keys in [lo, hi).
template <int NS, int NT, int MT, bool MASKED>
__device__ __forceinline__ void softmax_step(float (&s)[NS][NT][4], const float2 (&sc)[NS][2], const float (&fac)[NT][2], int key, const int (&lo)[NT][2],
                                             const int (&hi)[NT][2], float (&m)[NT][2], float (&l)[NT][2], float (&o)[NT][MT][4], uint32_t (&pb)[NS][NT][4]) {
  float lv[NS][2];  // exponents of the V scales (2^e <= scale < 2^(e + 1)), less the headroom
#pragma unroll
  for (int n = 0; n < NS; ++n)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float e = __uint_as_float((__float_as_uint(sc[n][i].y) >> 23) | 0x4b000000u) - (8388735.f + kHeadroom);
      lv[n][i] = e < 128.f - kHeadroom ? fmaxf(e, kLeastLog2 - kHeadroom) : -kHeadroom;
    }
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    bool see[NS][4];
    float top[2] = {-INFINITY, -INFINITY};
#pragma unroll
    for (int n = 0; n < NS; ++n)
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        see[n][c] = true;
        if constexpr (MASKED) {
          const int k = key + 16 * n + 8 * (c >> 1);
          see[n][c] = k >= lo[j][c & 1] && k < hi[j][c & 1];
        }
        s[n][j][c] = see[n][c] ? s[n][j][c] * (sc[n][c >> 1].x * fac[j][c & 1]) : -INFINITY;
        top[c & 1] = fmaxf(top[c & 1], see[n][c] ? s[n][j][c] + lv[n][c >> 1] : -INFINITY);
      }
    // (the first tile's maxima are above -inf + 8)
    if (__any_sync(0xffffffffu, top[0] > m[j][0] + 8.f || top[1] > m[j][1] + 8.f)) {
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        float mx = fmaxf(top[c], m[j][c]);
#pragma unroll
        for (int w = 4; w < 32; w <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
        const float f = shift2(m[j][c], mx);
        m[j][c] = mx;
        l[j][c] *= f;
#pragma unroll
        for (int i = 0; i < MT; ++i) o[j][i][c] *= f, o[j][i][c + 2] *= f;
      }
    }
    const float ref[2] = {MASKED && m[j][0] == -INFINITY ? 0.f : m[j][0], MASKED && m[j][1] == -INFINITY ? 0.f : m[j][1]};
#pragma unroll
    for (int n = 0; n < NS; ++n) {
      float wt[4];
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const float ex = see[n][c] ? tc::fast_exp2(s[n][j][c] - ref[c & 1]) : 0.f;
        l[j][c & 1] += ex;
        wt[c] = see[n][c] ? ex * sc[n][c >> 1].y : 0.f;
      }
      // A weight enters the products as its fp16 value and what that leaves over (2^-22 of it in all): rounded
      // once, a row with few keys would be 2^-11 off. The products are not what bounds this kernel.
#pragma unroll
      for (int c = 0; c < 4; c += 2) {
        const uint32_t h = tc::pack_half2(wt[c], wt[c + 1]);
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
        pb[n][j][c >> 1] = transpose8x8(h);
        pb[n][j][2 + (c >> 1)] = transpose8x8(tc::pack_half2(wt[c] - f.x, wt[c + 1] - f.y));
      }
    }
  }
}

// Groups of 16 keys of a tile: two chains where the accumulators leave registers for them.
template <int NT>
constexpr int kGroups = NT == 4 ? 1 : 2;
template <int DH, int BITS, int NT>
constexpr int kKeysSmem = W * DEPTH * Tile<DH, BITS, kGroups<NT>>::BYTES;

// Copies the key tiles of a warp's share of the list, one after the other, across items: the queue does not run dry
// between them.
template <int R, int KT>
struct Copier {
  static constexpr int NS = KT / 16, BATCH = 32 / NS;
  Item it;
  int64_t x, x1;       // tiles of the list
  int s, ready, places;  // tile of the item; tiles whose places are known; group lane % NS of tile lane / NS of those
  const int32_t* table;

  __device__ __forceinline__ void open(const AttnParams& p, const int* cum_t, const int* head) {
    it = item_at<R, KT>(p, cum_t, head, x, x1);
    s = it.s0;
    ready = 0;
    table = p.pages + (it.en.all ? 0 : (int64_t)(it.e - (p.list.all ? 1 : 0)) * p.max_pages);
  }
  // Places of the next tile's groups in the cache, in groups of 16 rows; false at the end of the share.
  __device__ __forceinline__ bool next(const AttnParams& p, const int* cum_t, const int* head, int lane, int (&rows)[NS]) {
    if (x >= x1) return false;
    if (s == it.s1) open(p, cum_t, head);
    if (ready == 0) {  // a lane finds one group's
      const int t = s + lane / NS, key = (it.t0 + t) * KT + (lane % NS) * 16;
      places = it.h * (p.page / 16);  // (past the keys there is nothing to see: any page, not the table's entry)
      if (t < it.s1 && key < it.en.len) {
        const int pg = p.by_page.quot(key);
        int id = __ldg(table + pg);
        if (id < 0 || id >= p.n_pages) {
          report(p.status, JAB_ERR_INVALID_ARG);
          id = 0;
        }
        places = (int)((((int64_t)id * p.n_kv + it.h) * p.page + (key - pg * p.page)) >> 4);
      }
      ready = BATCH;
    }
#pragma unroll
    for (int n = 0; n < NS; ++n) rows[n] = __shfl_sync(0xffffffffu, places, (BATCH - ready) * NS + n);
    --ready;
    ++s;
    ++x;
    return true;
  }
};

// Every warp works by itself on a share of its own.
template <class T, int DH, int BITS, int NT>
__global__ void __launch_bounds__(32 * W) kv_attn_kernel(const __grid_constant__ AttnParams p) {
  constexpr int R = 8 * NT, MT = DH / 16, KS = DH / 16, NS = kGroups<NT>, KT = 16 * NS;
  using TT = Tile<DH, BITS, NS>;
  extern __shared__ __align__(128) uint8_t dyn[];
  __shared__ int head[kPlanHead];
  const int E = entries(p);
  int* cum_t = reinterpret_cast<int*>(dyn + kKeysSmem<DH, BITS, NT>);
  int* cum_i = cum_t + E + 1;
  stream_order();
  make_plan<R, KT, W>(p, gridDim.x * W, cum_t, cum_i, head);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, q4 = lane & 3;
  const int worker = blockIdx.x * W + warp;
  const int64_t all = (int64_t)head[kTotal] * p.n_kv;
  const int64_t x0 = min((int64_t)worker * head[kPer], all), x1 = min(all, x0 + head[kPer]);
  uint8_t* queue = dyn + warp * DEPTH * TT::BYTES;
  const CopyLane<DH, BITS, NS> lanes(p, lane, tc::smem_u32(queue));
  Copier<R, KT> copier;
  copier.x = x0, copier.x1 = x1;
  copier.s = copier.it.s1 = 0;
  auto copy_next = [&](int slot) {
    int rows[NS];
    if (copier.next(p, cum_t, head, lane, rows)) lanes.copy(p, rows, lane, slot * TT::BYTES);
    copies_commit();
  };
#pragma unroll 1
  for (int d = 0; d < DEPTH; ++d) copy_next(d);
  int slot_q = 0;
  for (int64_t x = x0; x < x1;) {
    const Item it = item_at<R, KT>(p, cum_t, head, x, x1);
    const Entry& en = it.en;
    const int h = it.h, rt = it.rt;
    // Q, and what its rows see; rows past the end see, with a Q of zeros, only keys that no mask could hide: what lies in
    // hidden places must not move the references that the rows of a warp change together
    int all_lo, all_hi, lo[NT][2], hi[NT][2];
    seen_by_all(p, en, rt * R, rt * R + it.rows, head, all_lo, all_hi);
    uint32_t qf[NT][DH / 8];
    float fac[NT][2], o[NT][MT][4] = {}, m[NT][2], l[NT][2];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
      const int r = 8 * j + g, rr = rt * R + r, i = p.by_g.quot(rr), token = en.tok0 + i;
      const int64_t q_at = (int64_t)token * p.ldq + (int64_t)(h * p.G + rr - i * p.G) * DH;
      const bool used = r < it.rows && in_bounds(q_at + DH - 1, rows_extent(p, p.ldq, DH), p.status);
      const float back = load_q<T, DH, BITS>(static_cast<const T*>(p.q) + q_at, q4, used, qf[j]) * p.scale_log2;
      int row_lo = 0, row_hi = 0;
      if (r < it.rows) seen_by_row(p, en, en.all ? position_of(p, token) : en.len - en.nq + i, row_lo, row_hi);
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        fac[j][c] = __shfl_sync(0xffffffffu, back, 8 * q4 + 4 * c);
        lo[j][c] = __shfl_sync(0xffffffffu, row_lo, 8 * q4 + 4 * c);
        hi[j][c] = __shfl_sync(0xffffffffu, row_hi, 8 * q4 + 4 * c);
        m[j][c] = -INFINITY, l[j][c] = 0.f;
      }
    }
    for (int t = it.s0; t < it.s1; ++t) {
      copies_wait<DEPTH - 1>();
      __syncwarp();
      const uint8_t* tile = queue + slot_q * TT::BYTES;
      float2 sc[NS][2];
#pragma unroll
      for (int n = 0; n < 2 * NS; ++n) sc[n >> 1][n & 1] = *reinterpret_cast<const float2*>(tile + TT::S_OFF + (g + 8 * n) * 8);
      // S^T = K Q^T
      float s[NS][NT][4] = {};
#pragma unroll
      for (int n = 0; n < NS; ++n) {
        uint32_t kc[2][TT::KB / 4];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int c = 0; c < TT::KB / TT::KU; ++c)
            take<TT::KU>(tile + n * TT::GROUP + TT::k_at(g + 8 * i, (c * 4 + q4) * TT::KU), kc[i] + c * (TT::KU / 4));
#pragma unroll
        for (int i = 0; i < KS; i += BITS == 8 ? 1 : 2) {
          if constexpr (BITS == 8) {
            uint32_t a[4];
            bytes_h2(kc[0][i], a[0], a[2]);
            bytes_h2(kc[1][i], a[1], a[3]);
#pragma unroll
            for (int j = 0; j < NT; ++j) mma(s[n][j], a, qf[j][2 * i], qf[j][2 * i + 1]);
          } else {
            uint32_t u[4], w[4];
            nibbles_h2(kc[0][i / 2], u);
            nibbles_h2(kc[1][i / 2], w);
            const uint32_t a0[4] = {u[0], w[0], u[1], w[1]}, a1[4] = {u[2], w[2], u[3], w[3]};
#pragma unroll
            for (int j = 0; j < NT; ++j) {
              mma(s[n][j], a0, qf[j][2 * i], qf[j][2 * i + 1]);
              mma(s[n][j], a1, qf[j][2 * i + 2], qf[j][2 * i + 3]);
            }
          }
        }
      }
      const int key0 = (it.t0 + t) * KT;
      uint32_t pb[NS][NT][4];
      if (key0 < all_lo || key0 + KT > all_hi)
        softmax_step<NS, NT, MT, true>(s, sc, fac, key0 + g, lo, hi, m, l, o, pb);
      else
        softmax_step<NS, NT, MT, false>(s, sc, fac, key0 + g, lo, hi, m, l, o, pb);
      // O^T += V^T P^T
#pragma unroll
      for (int n = 0; n < NS; ++n) {
        uint32_t vc[4][TT::VB / 4];
#pragma unroll
        for (int i = 0; i < 4; ++i) take<TT::VB>(tile + TT::V_OFF + n * TT::GROUP + TT::v_at(4 * i + q4, g * TT::VB), vc[i]);
#pragma unroll
        for (int w = 0; w < TT::VB / 4; ++w) {
          uint32_t ab[2][2];  // [keys 2q.. / 2q + 8..]: dimensions interleaved, pairs of keys
          if constexpr (BITS == 8) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              ab[i][0] = __byte_perm(vc[2 * i][w], vc[2 * i + 1][w], 0x5140);  // a0 b0 a1 b1
              ab[i][1] = __byte_perm(vc[2 * i][w], vc[2 * i + 1][w], 0x7362);  // a2 b2 a3 b3
            }
#pragma unroll
            for (int d = 0; d < 2; ++d) {
              uint32_t a[4];
              bytes_h2(ab[0][d], a[0], a[1]);
              bytes_h2(ab[1][d], a[2], a[3]);
#pragma unroll
              for (int j = 0; j < NT; ++j) {
                mma(o[j][2 * w + d], a, pb[n][j][0], pb[n][j][1]);
                mma(o[j][2 * w + d], a, pb[n][j][2], pb[n][j][3]);
              }
            }
          } else {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              ab[i][0] = __byte_perm(vc[2 * i][w], vc[2 * i + 1][w], 0x5410);  // low halves
              ab[i][1] = __byte_perm(vc[2 * i][w], vc[2 * i + 1][w], 0x7632);  // high halves
            }
#pragma unroll
            for (int d = 0; d < 2; ++d) {
              uint32_t u[4], x2[4];
              nibbles_h2(ab[0][d], u);
              nibbles_h2(ab[1][d], x2);
              const uint32_t a0[4] = {u[0], u[1], x2[0], x2[1]}, a1[4] = {u[2], u[3], x2[2], x2[3]};
#pragma unroll
              for (int j = 0; j < NT; ++j) {
                mma(o[j][4 * w + 2 * d], a0, pb[n][j][0], pb[n][j][1]);
                mma(o[j][4 * w + 2 * d + 1], a1, pb[n][j][0], pb[n][j][1]);
                mma(o[j][4 * w + 2 * d], a0, pb[n][j][2], pb[n][j][3]);
                mma(o[j][4 * w + 2 * d + 1], a1, pb[n][j][2], pb[n][j][3]);
              }
            }
          }
        }
      }
      __syncwarp();  // all lanes have read the tile
      copy_next(slot_q);
      slot_q = slot_q + 1 == DEPTH ? 0 : slot_q + 1;
    }
    // the item's rows: output, or a part. A lane has DH / 8 dimensions of rows 8j + 2q, 8j + 2q + 1.
    const bool whole = it.s0 == 0 && it.s1 == it.n && p.shared == 0;
    const int64_t slot = slot_of(p, worker, h * head[kItems] + cum_i[it.e] + rt, x == x0);
    if (!whole && slot >= p.list.n_slots) report(p.status, JAB_ERR_INVALID_ARG);
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
#pragma unroll
        for (int w = 4; w < 32; w <<= 1) l[j][c] += __shfl_xor_sync(0xffffffffu, l[j][c], w);
        const int r = 8 * j + 2 * q4 + c, rr = rt * R + r, i = p.by_g.quot(rr), qh = h * p.G + rr - i * p.G;
        const int64_t token = en.tok0 + i;
        if (r >= it.rows) continue;
        if (whole) {
          const float inv = l[j][c] == 0.f ? 0.f : 1.f / l[j][c];
          const int64_t at = token * p.ldo + (int64_t)qh * DH + g * (DH / 8), lse_at = token * ((int64_t)p.n_kv * p.G) + qh;
          T* out = static_cast<T*>(p.out) + at;
#pragma unroll
          for (int d = 0; d < MT; d += 4) {
            __align__(16) T v[8];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              store_out(v + 2 * k, o[j][d + k][c] * inv);
              store_out(v + 2 * k + 1, o[j][d + k][c + 2] * inv);
            }
            if (out_fits(p, at + 2 * d + 7, DH)) *reinterpret_cast<uint4*>(out + 2 * d) = *reinterpret_cast<const uint4*>(v);
          }
          if (g == 0 && p.lse != nullptr && lse_fits(p, lse_at))
            p.lse[lse_at] = l[j][c] == 0.f ? -INFINITY : (m[j][c] + log2f(l[j][c])) * kLn2;
        } else if (slot < p.list.n_slots && part_fits(p, (slot * R + r + 1) * DH - 1, R, DH)) {
          float* part = p.list.part_o + (slot * R + r) * DH + g * (DH / 8);
#pragma unroll
          for (int d = 0; d < MT; d += 2)
            *reinterpret_cast<float4*>(part + 2 * d) = make_float4(o[j][d][c], o[j][d][c + 2], o[j][d + 1][c], o[j][d + 1][c + 2]);
          if (g == 0) p.list.part_ml[slot * R + r] = make_float2(m[j][c], l[j][c]);
        }
      }
    x += it.s1 - it.s0;
  }
  copies_wait<0>();
}

// ------------------------------------------------------------------ joining
// N floats at p (N 2 or 4) if `there`, else zeros; not from this SM's cache: other SMs wrote them. (volatile: a batch of
// them is under way at once. Reading some one place instead of none would bring all SMs to the same line.)
template <int N>
__device__ __forceinline__ void load_part(const float* p, bool there, float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) v[i] = 0.f;
  if constexpr (N == 4)
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %5, 0;\n\t@q ld.global.cg.v4.f32 {%0, %1, %2, %3}, [%4];\n\t}"
                 : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]) : "l"(p), "r"((int)there));
  else
    asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %3, 0;\n\t@q ld.global.cg.v2.f32 {%0, %1}, [%2];\n\t}"
                 : "+f"(v[0]), "+f"(v[1]) : "l"(p), "r"((int)there));
}

constexpr int MW = 8;  // warps of a joining block

// A list as the joining kernel needs it.
struct Joined {
  const int32_t* plan;
  const int4* items;
  const float2* part_ml;
  const float* part_o;
  int n_slots, max_items, rows, groups;  // rows of an item, groups of MW rows of an item
  bool all;
};

// Joins the parts of the rows whose keys went to several workers or entries, in a fixed order: a block per KV head (y) and
// MW rows of an item (x), of list 0 (kv_attn_kernel's), then of list 1 (the tile kernel's); a list that was not run has
// no items. A trip to memory that other SMs wrote takes 0.6 us here, so that what counts is their number: the plan and
// the item's record, then statistics and rows of BATCH parts at once. (One block per item over a chain of five trips took
// 13 us for 64 sequences of up to 8192 keys.)
// BATCH: parts of a row on their way at once; 16 for calls with few rows, which have many parts (4 sequences of 65536
// keys: 73 us in all, 88 with 4), 4 where many blocks an SM are worth more (2 x 512 queries behind 5000 keys: 150, 159 with
// 16; in between the difference is small and the other way: 64 behind a shared prefix of 8192 67.6, 65.2 with 16).
template <class T, int DH, int BATCH>
__global__ void __launch_bounds__(32 * MW, BATCH == 4 ? 6 : 2)
    kv_merge_kernel(const __grid_constant__ AttnParams p, const __grid_constant__ Joined j0, const __grid_constant__ Joined j1) {
  constexpr int N = DH / 32;  // dimensions of a lane
  __shared__ float2 sm_ml[MW];
  __shared__ float sm_o[MW][DH];
  stream_order();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, h = blockIdx.y;
  const bool first_list = blockIdx.x < (unsigned)(j0.max_items * j0.groups);
  const Joined own = first_list ? j0 : j1, common = j1.all ? j1 : j0;  // (common: where the shared keys' entry is)
  const int u = first_list ? blockIdx.x : blockIdx.x - j0.max_items * j0.groups, i = u / own.groups, r0 = (u - i * own.groups) * MW;
  const int4 it = __ldcg(own.items + i);
  const int items = __ldcg(own.plan + kItems), per = __ldcg(own.plan + kPer), total = __ldcg(own.plan + kTotal);
  int4 it_c = make_int4(0, 0, 0, 1);
  int items_c = 0, per_c = 1, total_c = 0;
  if (p.shared > 0) {
    it_c = __ldcg(common.items);
    items_c = __ldcg(common.plan + kItems), per_c = __ldcg(common.plan + kPer), total_c = __ldcg(common.plan + kTotal);
  }
  if (i >= items || (p.shared > 0 && items_c == 0)) return;  // (a list too long to be run is empty)
  // (the shared keys' own items are taken with the sequences')
  if (own.all && i < ((int64_t)p.n_tokens * p.G + own.rows - 1) / own.rows) return;
  const int rt = it.y >> 8, rows = min((it.y & 255) - r0, MW);
  const int64_t y0 = (int64_t)h * total + it.z;
  if (rows <= 0 || (p.shared == 0 && (int)(y0 / per) == (int)((y0 + it.w - 1) / per))) return;  // (written by its worker)
  // several warps to a row where there are few
  int ways = 1;
  while (2 * ways * rows <= MW) ways *= 2;
  const int way = warp & (ways - 1), r = r0 + warp / ways;
  const bool live = r < r0 + rows;
  const int rr = rt * own.rows + r, q = p.by_g.quot(rr), token = it.x + q, qh = h * p.G + rr - q * p.G;
  float mx = -INFINITY, l = 0.f, o[N] = {};
#pragma unroll 1
  for (int k = p.shared > 0 ? 0 : 1; k < 2 && live; ++k) {
    // the shared keys' entry (the first of its list), then the item itself
    const Joined& list = k == 0 ? common : own;
    int item = i, row = r, n = it.w, each = per;
    int64_t y = y0;
    if (k == 0) {
      const int all_row = token * p.G + rr - q * p.G;
      item = all_row / common.rows;
      row = all_row - item * common.rows;
      n = it_c.w;
      y = (int64_t)h * total_c + (int64_t)item * n;
      each = per_c;
    }
    item += h * (k == 0 ? items_c : items);
    const int first = (int)(y / each), last = (int)((y + n - 1) / each), share = (last - first + ways) / ways;
    const int c0 = first + way * share, c1 = min(c0 + share - 1, last);
#pragma unroll 1
    for (int c = c0; c <= c1; c += BATCH) {
      const int mine = c + (lane & (BATCH - 1));
      const int64_t slot = slot_of(p, mine, item, (int64_t)mine * each >= y);
      const bool have = mine <= c1 && slot < list.n_slots;
      float v[BATCH][N];
#pragma unroll
      for (int b = 0; b < BATCH; ++b) {
        const int64_t at = slot_of(p, c + b, item, (int64_t)(c + b) * each >= y);
        load_part<N>(list.part_o + (at * list.rows + row) * DH + lane * N, c + b <= c1 && at < list.n_slots, v[b]);
      }
      const float2 ml = have ? __ldcg(list.part_ml + slot * list.rows + row) : make_float2(-INFINITY, 0.f);
      float mn = ml.x;
#pragma unroll
      for (int w = BATCH / 2; w > 0; w >>= 1) mn = fmaxf(mn, __shfl_xor_sync(0xffffffffu, mn, w));
      mn = fmaxf(mn, mx);
      const float f = shift2(ml.x, mn), fa = shift2(mx, mn);
      float add = ml.y * f;
#pragma unroll
      for (int w = BATCH / 2; w > 0; w >>= 1) add += __shfl_xor_sync(0xffffffffu, add, w);
      mx = mn;
      l = l * fa + add;
#pragma unroll
      for (int d = 0; d < N; ++d) o[d] *= fa;
#pragma unroll
      for (int b = 0; b < BATCH; ++b) {
        const float fk = __shfl_sync(0xffffffffu, f, b);
#pragma unroll
        for (int d = 0; d < N; ++d) o[d] += fk == 0.f ? 0.f : fk * v[b][d];
      }
    }
  }
  if (ways > 1) {
    if (lane == 0) sm_ml[warp] = make_float2(mx, l);
#pragma unroll
    for (int d = 0; d < N; ++d) sm_o[warp][lane * N + d] = o[d];
    __syncthreads();
    if (way > 0) return;
    mx = -INFINITY;
#pragma unroll 1
    for (int w = 0; w < ways; ++w) mx = fmaxf(mx, sm_ml[warp + w].x);
    l = 0.f;
#pragma unroll
    for (int d = 0; d < N; ++d) o[d] = 0.f;
#pragma unroll 1
    for (int w = 0; w < ways; ++w) {
      const float f = shift2(sm_ml[warp + w].x, mx);
      l += f * sm_ml[warp + w].y;
#pragma unroll
      for (int d = 0; d < N; ++d) o[d] += f * sm_o[warp + w][lane * N + d];
    }
  }
  if (!live) return;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  const int64_t at = (int64_t)token * p.ldo + (int64_t)qh * DH + lane * N, lse_at = (int64_t)token * (p.n_kv * p.G) + qh;
  if (!out_fits(p, at + N - 1, DH) || !lse_fits(p, lse_at)) return;
  T* out = static_cast<T*>(p.out) + at;
  __align__(8) T v[N];
#pragma unroll
  for (int d = 0; d < N; ++d) store_out(v + d, o[d] * inv);
  if constexpr (N == 4)
    *reinterpret_cast<uint2*>(out) = *reinterpret_cast<const uint2*>(v);
  else
    *reinterpret_cast<uint32_t*>(out) = *reinterpret_cast<const uint32_t*>(v);
  if (lane == 0 && p.lse != nullptr) p.lse[lse_at] = l == 0.f ? -INFINITY : (mx + log2f(l)) * kLn2;
}

// ------------------------------------------------------------------ host side
constexpr int kMaxBlocks = 608, kMaxTileBlocks = 512;  // (workers of the by-keys kernel: W times as many)
constexpr int kFewRows = 32;   // rows of a sequence up to which all of the work goes by 16 keys
constexpr int kFewBeside = 16;  // the same where longer ones are in the batch

int n_tiles_of_rows(int64_t rows) { return rows <= 8 ? 1 : rows <= 16 ? 2 : 4; }

// Which kernel takes what. Sequences of up to kFewRows (token, head) rows go by 16-key tiles: the cache's bytes bound
// them, not the products. Longer ones fill 128-row tiles; where lengths are mixed, those of up to kFewBeside rows still go
// by keys, in a launch of their own. Measured, both ways (heads of 128, 8 bits, G = 4, 300 to 2048 keys): 64 sequences of 16
// rows 53 us by keys and 135 by tiles, of 32 rows 96 and 138, of 36 rows 143 and 139, of 64 rows 157 and 143; 4 of 32
// behind 8192 keys 54 and 49, of 36 69 and 49. (With heads of 64 and G = 1 the bound would lie higher: 64 sequences of 40 rows
// 135 and 181, but 4 of 40 behind 8192 keys 64 and 53.) Beside a chunk of 512 tokens, with bounds of 8, 16 and 32 (G = 4, up to 2048
// keys): 64 sequences of 4 rows 101, 104 and 149 us, of 16 rows 192, 110 and 156, of 32 rows 195, 197 and 166; with up to
// 8192 keys 4 rows 131, 139 and 244, 16 rows 276, 147 and 254; single tokens at G = 16 100, 84 and 98. (Rows of one tile wait for
// the longest of them: a bound of 16 makes all of them 16.)
struct Route {
  List keys, tiles;
  int nt;  // 8-row blocks of the by-keys kernel
  size_t keys_plan, keys_items, keys_ml, keys_o, tiles_plan, tiles_items, tiles_ml, tiles_o, total;
};

Route route(int dh, int n_kv, int n_seqs, int64_t n_tokens, int G, int max_q, bool shared) {
  Route r{};
  const int64_t rows = (int64_t)max_q * G, all_rows = n_tokens * G;
  const bool tiles_own = rows > kFewRows, uniform = n_tokens == (int64_t)n_seqs * max_q;
  const bool tiles_all = shared && all_rows > kFewRows;
  const bool keys_own = !tiles_own || !uniform, keys_all = shared && !tiles_all;
  r.keys.used = keys_own || keys_all;
  r.tiles.used = tiles_own || tiles_all;
  r.keys.all = keys_all;
  r.tiles.all = tiles_all;
  r.nt = !tiles_own ? n_tiles_of_rows(keys_all ? std::max(rows, all_rows) : rows) : keys_all ? 4 : n_tiles_of_rows(kFewBeside);
  const int split = !tiles_own ? INT32_MAX : uniform ? 0 : kFewBeside;  // rows up to which a sequence goes by keys
  r.keys.min_rows = 1, r.keys.max_rows = keys_own ? split : 0;
  r.tiles.min_rows = tiles_own ? split + 1 : INT32_MAX, r.tiles.max_rows = INT32_MAX;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t o = at;
    at = (at + bytes + 255) / 256 * 256;
    return o;
  };
  auto slots = [&](int blocks, int R, bool all, bool own) {
    if (!shared) return 2 * (int64_t)blocks;
    return blocks + (int64_t)n_kv * ((all ? (all_rows + R - 1) / R : 0) + (own ? (all_rows + R - 1) / R + n_seqs : 0));
  };
  const size_t plan_bytes = kPlanHead * 4;
  auto items = [&](int R, bool all, bool own) {
    const int64_t n = (all ? (all_rows + R - 1) / R : 0) + (own ? (all_rows + R - 1) / R + n_seqs : 0);
    return (int)std::min<int64_t>(n, INT32_MAX);
  };
  if (r.keys.used) {
    const int R = 8 * r.nt;
    const int64_t n = slots(kMaxBlocks * W, R, keys_all, keys_own);
    r.keys.n_slots = (int)std::min<int64_t>(n, INT32_MAX);
    r.keys.max_items = items(R, keys_all, keys_own);
    r.keys_plan = take(plan_bytes), r.keys_items = take((size_t)r.keys.max_items * 16), r.keys_ml = take((size_t)n * R * 8), r.keys_o = take((size_t)n * R * dh * 4);
  }
  if (r.tiles.used) {
    const int64_t n = slots(kMaxTileBlocks, kTileRows, tiles_all, tiles_own);
    r.tiles.n_slots = (int)std::min<int64_t>(n, INT32_MAX);
    r.tiles.max_items = items(kTileRows, tiles_all, tiles_own);
    r.tiles_plan = take(plan_bytes), r.tiles_items = take((size_t)r.tiles.max_items * 16), r.tiles_ml = take((size_t)n * kTileRows * 8), r.tiles_o = take((size_t)n * kTileRows * dh * 4);
  }
  r.total = std::max<size_t>(at, 256);
  return r;
}

template <class T, int DH, int BITS, int NT>
cudaError_t launch_keys(const AttnParams& p, int64_t est_tiles, int sms, cudaStream_t st) {
  auto kern = kv_attn_kernel<T, DH, BITS, NT>;
  const size_t most = kKeysSmem<DH, BITS, NT> + (size_t)2 * (2048 + 2) * 4;
  static SetUp ready;
  static Found resident;  // blocks an SM, by the number of entries
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  e = ready.once(dev, [&] { return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most); });
  if (e != cudaSuccess) return e;
  const int E = p.n_seqs + (p.list.all ? 1 : 0);
  const size_t smem = kKeysSmem<DH, BITS, NT> + (size_t)2 * (E + 1) * 4;
  const int occ = resident.get(dev, E, [&] {
    int n = 0;
    e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&n, kern, 32 * W, smem);
    return e == cudaSuccess ? std::max(n, 1) : 0;
  });
  if (e != cudaSuccess) return e;
  const int64_t grid = std::max<int64_t>(1, std::min<int64_t>({(int64_t)sms * occ, kMaxBlocks, (est_tiles + W - 1) / W}));
  return launch_after(kern, (unsigned)grid, 32 * W, smem, st, p);
}

// Tiles that a launch has at most, by the caller's hints, which may be as large as their types hold.
int64_t estimate(double tiles) { return (int64_t)std::min(tiles, 1e15); }

template <class T, int DH>
cudaError_t launch_all(AttnParams p, const Route& r, int bits, jab_dtype type, int max_q, int max_len, int sms, cudaStream_t st) {
  cudaError_t e;
  if (r.keys.used) {
    p.list = r.keys;
    const int64_t est = estimate((double)p.n_kv * p.n_seqs * (max_len / 32 + 1) * std::max<int64_t>(1, (int64_t)max_q * p.G / (8 * r.nt)));
    if (bits == 8)
      e = r.nt == 1 ? launch_keys<T, DH, 8, 1>(p, est, sms, st) : r.nt == 2 ? launch_keys<T, DH, 8, 2>(p, est, sms, st) : launch_keys<T, DH, 8, 4>(p, est, sms, st);
    else
      e = r.nt == 1 ? launch_keys<T, DH, 4, 1>(p, est, sms, st) : r.nt == 2 ? launch_keys<T, DH, 4, 2>(p, est, sms, st) : launch_keys<T, DH, 4, 4>(p, est, sms, st);
    if (e != cudaSuccess) return e;
  }
  if (r.tiles.used) {
    p.list = r.tiles;
    p.behind = r.keys.used;
    const int64_t rts = ((int64_t)max_q * p.G + kTileRows - 1) / kTileRows, kts = max_len / kTileKeys + 1;
    const int64_t est = estimate(p.n_kv * ((double)p.n_seqs * rts * kts + (r.tiles.all ? ((double)p.n_tokens * p.G / kTileRows + 1) * kts : 0)));
    if ((e = launch_tiles(p, type, DH, bits, est, std::min(sms, kMaxTileBlocks), st)) != cudaSuccess) return e;
  }
  auto joined = [](const List& l, int rows) {
    Joined j{l.plan, l.items, l.part_ml, l.part_o, l.n_slots, l.used ? l.max_items : 0, rows, (rows + MW - 1) / MW, l.used && l.all};
    return j;
  };
  const Joined j0 = joined(r.keys, 8 * r.nt), j1 = joined(r.tiles, kTileRows);
  cudaLaunchConfig_t cfg = {};
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.gridDim = dim3((unsigned)(j0.max_items * j0.groups + j1.max_items * j1.groups), (unsigned)p.n_kv);
  cfg.blockDim = dim3(32 * MW);
  cfg.stream = st;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  e = cfg.gridDim.x * cfg.gridDim.y <= 2u * (unsigned)sms ? cudaLaunchKernelEx(&cfg, kv_merge_kernel<T, DH, 16>, p, j0, j1)
                                                          : cudaLaunchKernelEx(&cfg, kv_merge_kernel<T, DH, 4>, p, j0, j1);
  if (e != cudaSuccess) cudaGetLastError();
  return e;
}

}  // namespace
}  // namespace kv

size_t kv_attention_scratch(int n_kv, int dh, int n_seqs, int64_t n_tokens, int n_q_heads, int max_q, int shared) {
  return kv::route(dh, n_kv, n_seqs, n_tokens, n_q_heads / n_kv, max_q, shared > 0).total;
}

int kv_attention_kernels(const KvAttnArgs& a) {
  const int n_kv = a.cache.n_kv_heads;
  const kv::Route r = kv::route(a.cache.head_dim, n_kv, a.n_seqs, a.n_tokens, a.n_q_heads / n_kv, a.max_q, a.shared > 0);
  return (r.keys.used ? 1 : 0) + (r.tiles.used ? 1 : 0) + 1;
}

cudaError_t launch_kv_attention(const KvAttnArgs& a, int sms, cudaStream_t st) {
  const jab_kv_cache& c = a.cache;
  kv::AttnParams p{};
  p.k_codes = static_cast<const uint8_t*>(c.k_codes);
  p.v_codes = static_cast<const uint8_t*>(c.v_codes);
  p.k_scales = c.k_scales;
  p.v_scales = c.v_scales;
  p.n_kv = c.n_kv_heads;
  p.G = a.n_q_heads / c.n_kv_heads;
  p.n_pages = (int)std::min<int64_t>(c.n_pages, INT32_MAX);
  p.max_pages = a.max_pages;
  p.page = c.page_tokens;
  p.copy_keys = std::min(c.page_tokens & -c.page_tokens, kv::kTileKeys);
  p.by_page = FastDiv(p.page);
  p.by_g = FastDiv(p.G);
  p.q = a.q;
  p.ldq = a.ldq;
  p.q_start = a.q_start;
  p.pages = a.pages;
  p.lens = a.lens;
  p.n_seqs = a.n_seqs;
  p.n_tokens = (int)a.n_tokens;
  p.shared = a.shared;
  p.window = a.window;
  p.scale_log2 = a.scale * kv::kLog2e;
  p.out = a.out;
  p.ldo = a.ldo;
  p.lse = a.lse;
  p.status = a.status;
  kv::Route r = kv::route(c.head_dim, p.n_kv, p.n_seqs, p.n_tokens, p.G, a.max_q, p.shared > 0);
  char* w = static_cast<char*>(a.ws);
  r.keys.plan = reinterpret_cast<int32_t*>(w + r.keys_plan);
  r.keys.items = reinterpret_cast<int4*>(w + r.keys_items);
  r.tiles.items = reinterpret_cast<int4*>(w + r.tiles_items);
  r.keys.part_ml = reinterpret_cast<float2*>(w + r.keys_ml);
  r.keys.part_o = reinterpret_cast<float*>(w + r.keys_o);
  r.tiles.plan = reinterpret_cast<int32_t*>(w + r.tiles_plan);
  r.tiles.part_ml = reinterpret_cast<float2*>(w + r.tiles_ml);
  r.tiles.part_o = reinterpret_cast<float*>(w + r.tiles_o);
  const bool wide = c.head_dim == 128;
  if (a.type == JAB_FP16)
    return wide ? kv::launch_all<half_t, 128>(p, r, c.bits, a.type, a.max_q, a.max_len, sms, st)
                : kv::launch_all<half_t, 64>(p, r, c.bits, a.type, a.max_q, a.max_len, sms, st);
  return wide ? kv::launch_all<bf16_t, 128>(p, r, c.bits, a.type, a.max_q, a.max_len, sms, st)
              : kv::launch_all<bf16_t, 64>(p, r, c.bits, a.type, a.max_q, a.max_len, sms, st);
}

}  // namespace jab
